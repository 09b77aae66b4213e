/*
 * im2win_seq.h -- operators over sequences of tokens: the short causal
 * convolution of state space layers (a depthwise convolution along time),
 * the selective state space scan that reads its output, and the
 * root-mean-square norm with the residual's addition in front of both; and
 * those of the layers that stand between such layers in hybrid stacks: the
 * gated linear recurrence, the norm of queries and keys with the position
 * rotation, and attention with a sliding window.
 * Exported by libim2win beside the im2win entry points of im2win.h (same
 * error codes, error messages and conventions about streams and ownership;
 * see there).  Where this header differs:
 *
 *  - Tokens are rows.  A tensor of T tokens and D channels is T x D with its
 *    channels contiguous; inputs may have a row stride of their own (ld_*, in
 *    elements, at least the row's width), so that slices of a wider row can
 *    be read in place.  Outputs are dense.
 *  - Sequences lie one behind the other in the rows.  seq_starts (device,
 *    sequences + 1 int32, not decreasing) gives their first rows: sequence b
 *    is [seq_starts[b], seq_starts[b+1]), possibly empty.  NULL means
 *    sequences of tokens / sequences rows each.  Rows before the first start
 *    and behind the last are neither read nor written.  Values outside of
 *    [0, tokens] are taken as the nearest of the two.
 *  - Pointers need the alignment of their element type only; workspaces need
 *    16 bytes.  Row strides stay below 2^28 elements.  Sizes whose launch would
 *    hold 2^32 threads (some 2^24 rows and more, of few channels) are refused
 *    with EOVERFLOW before anything is launched; the norm takes them.
 *  - Arrays of T rows may be NULL when tokens is 0.  Outputs must not overlap
 *    inputs or each other, except where an entry point says so.
 *  - "dtype" arrays hold im2win_dtype elements; every sum, state, statistic
 *    and gradient of a parameter is fp32.  Results are rounded once, when
 *    they are written, and every sum has a fixed order: a call gives the same
 *    bits each time.
 */
#ifndef IM2WIN_SEQ_H
#define IM2WIN_SEQ_H

#include "im2win.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------------------------ */
/* Short causal convolution                                                  */
/* ------------------------------------------------------------------------ */

typedef struct {
    int64_t tokens;      /* T, rows of x (requests, for the step) */
    int64_t channels;    /* D */
    int64_t width;       /* W, taps, 1 to 8 */
    int64_t sequences;   /* B >= 1 (not used by the step) */
    int64_t ld_x;        /* row stride of x */
    int32_t dtype;       /* of x, w, bias, y, the states and their gradients */
    int32_t silu;        /* nonzero: y = s * sigmoid(s) of the sum s */
} im2win_conv1d_desc;

/*
 * y[t][c] = act(bias[c] + sum_{k<W} w[c][k] * x[t - (W-1) + k][c])
 * where the inputs before a sequence's first row are its initial state's
 * rows (initial_state[b][j] lies W-1-j tokens before the first), or zero.
 *   x              device, T x D, row stride ld_x
 *   w              device, D x W;  bias  device, D, or NULL
 *   initial_state  device, B x (W-1) x D, or NULL (zeros)
 *   y              device, T x D
 *   final_state    device, B x (W-1) x D, or NULL: the last W-1 inputs of
 *                  each sequence (of its initial state too, where it is
 *                  shorter), as the next call's initial state
 * Errors: EINVAL, ENULL, EALIGN, EOVERFLOW, EHIP.
 */
int im2win_causal_conv1d(const im2win_conv1d_desc* d, const void* x, const void* w,
                         const void* bias, const int32_t* seq_starts, const void* initial_state,
                         void* y, void* final_state, void* stream);

/* Bytes of workspace that im2win_causal_conv1d_backward takes.  Host only. */
int im2win_causal_conv1d_backward_workspace_bytes(const im2win_conv1d_desc* d, size_t* bytes);

/*
 * Gradients of im2win_causal_conv1d for the gradient dy of y (T x D) and,
 * where d_final_state (B x (W-1) x D) is given, of the final state.
 *   dx               device, T x D
 *   dw, dbias        device, D x W and D, fp32 (dbias may be NULL)
 *   d_initial_state  device, B x (W-1) x D, or NULL
 *   workspace        device, 16-byte aligned, at least the bytes above
 * Errors: EINVAL, ENULL, EALIGN, EWORKSPACE, EOVERFLOW, EHIP.
 */
int im2win_causal_conv1d_backward(const im2win_conv1d_desc* d, const void* dy, const void* x,
                                  const void* w, const void* bias, const int32_t* seq_starts,
                                  const void* initial_state, const void* d_final_state, void* dx,
                                  float* dw, float* dbias, void* d_initial_state, void* workspace,
                                  size_t workspace_bytes, void* stream);

/*
 * One token for each of d->tokens requests.  Request i's last W-1 inputs are
 * state[slots[i]] of a pool of state_slots states (W-1 x D each); the call
 * moves them on by one token in place.  slots NULL means slot i.  A request
 * whose slot is outside of [0, state_slots) gets y = 0 and leaves the pool as
 * it is.  No two requests may name the same slot.
 *   x, y   device, T x D (x with row stride ld_x);  w, bias as above
 *   state  device, state_slots x (W-1) x D (read and written; may be NULL
 *          when W is 1)
 * Errors: EINVAL, ENULL, EALIGN, EOVERFLOW, EHIP.
 */
int im2win_causal_conv1d_step(const im2win_conv1d_desc* d, const void* x, const void* w,
                              const void* bias, const int32_t* slots, void* state,
                              int64_t state_slots, void* y, void* stream);

/* ------------------------------------------------------------------------ */
/* Root-mean-square norm with the residual's addition                        */
/* ------------------------------------------------------------------------ */

typedef struct {
    int64_t tokens;          /* T */
    int64_t channels;        /* D, at most 16384 */
    int64_t ld_x;            /* row stride of x */
    int64_t block;           /* channels that share a scale of the 8-bit output: 0 (the row), or a
                                power of two from 16 to 512 that divides D */
    int32_t dtype;           /* of x, y and dy */
    int32_t residual_dtype;  /* of the residual, h and their gradients */
    float eps;               /* >= 0 */
} im2win_norm_desc;

/*
 * h[t] = x[t] + residual[t], rounded to residual_dtype (h = x so rounded
 * where residual is NULL);
 * y[t][c] = h[t][c] * rsqrt(mean_c(h[t][c]^2) + eps) * w[c], of the rounded h.
 *   x         device, T x D, row stride ld_x
 *   residual  device, T x D, or NULL
 *   w         device, D, fp32
 *   y         device, T x D
 *   h         device, T x D; may be residual itself (the sum in place), and
 *             may be NULL where residual is NULL
 * Errors: EINVAL, ENULL, EALIGN, EOVERFLOW, EHIP.
 */
int im2win_add_rms_norm(const im2win_norm_desc* d, const void* x, const void* residual, const float* w,
                        void* y, void* h, void* stream);

/*
 * The same with y in 8 bits (OCP e4m3: 4 bits of exponent, 3 of mantissa,
 * largest value 448): for each row, or each `block` channels of it,
 *   scale = max |y| / 448 (1 where that is 0 in fp32, as in a block of zeros,
 *   or where the block holds a NaN),
 *   q = y / scale, rounded to nearest even.  y is not rounded before.  Where
 *   the scale is subnormal, and so rounded coarsely, quotients beyond 448 are
 *   taken as 448.  Beside a NaN in its block a y beyond 448 has no value in q.
 *   q       device, T x D, one byte each
 *   scales  device, T x (D / block) (T x 1 for block 0), fp32
 * Errors: EINVAL, ENULL, EALIGN, EOVERFLOW, EHIP.
 */
int im2win_add_rms_norm_fp8(const im2win_norm_desc* d, const void* x, const void* residual, const float* w,
                            void* q, float* scales, void* h, void* stream);

/* Bytes of workspace that im2win_add_rms_norm_backward takes.  Host only. */
int im2win_add_rms_norm_backward_workspace_bytes(const im2win_norm_desc* d, size_t* bytes);

/*
 * Gradients for dy (T x D) and, where it is given, d_residual (T x D, the
 * gradient that h receives from elsewhere): with r = rsqrt(mean(h^2) + eps)
 * and g = dy w,
 *   dx = r (g - h r^2 mean(g h)) + d_residual,  the gradient of x and of residual,
 *   dw[c] = sum_t dy[t][c] h[t][c] r[t].
 *   h   device, T x D, as the forward call wrote it
 *   dx  device, T x D, residual_dtype; may be d_residual itself
 *   dw  device, D, fp32
 *   workspace  device, 16-byte aligned, at least the bytes above
 * Errors: EINVAL, ENULL, EALIGN, EWORKSPACE, EOVERFLOW, EHIP.
 */
int im2win_add_rms_norm_backward(const im2win_norm_desc* d, const void* dy, const void* h, const float* w,
                                 const void* d_residual, void* dx, float* dw, void* workspace,
                                 size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------ */
/* Selective state space scan                                                */
/* ------------------------------------------------------------------------ */

typedef struct {
    int64_t tokens;      /* T (requests, for the step) */
    int64_t channels;    /* D */
    int64_t states;      /* N, states of a channel, 1 to 128 */
    int64_t groups;      /* G: channel c reads B and C of group c / (D / G); divides D */
    int64_t sequences;   /* S >= 1 (not used by the step) */
    int64_t ld_x, ld_dt, ld_z;   /* row strides of x, dt and z */
    int64_t ld_b, ld_c;          /* row strides of B and C (rows of G x N) */
    int32_t dtype;       /* of x, dt, B, C, z, y and their gradients */
    int32_t softplus;    /* nonzero: the step size is log(1 + exp(dt + dt_bias)) */
} im2win_scan_desc;

/*
 * For each channel c and state n, along each sequence,
 *   s[t][c]    = act(dt[t][c] + dt_bias[c])
 *   h[t][c][n] = exp(s[t][c] A[c][n]) h[t-1][c][n] + s[t][c] x[t][c] B[t][g(c)][n]
 *   y[t][c]    = (sum_n C[t][g(c)][n] h[t][c][n] + D[c] x[t][c]) * z[t][c] sigmoid(z[t][c])
 * where the state before a sequence is its initial state, or zero.  Behind an
 * infinite or NaN x or step its channel has no finite values up to the
 * sequence's end (where the formula gives infinities, NaN may stand).
 *   x, dt     device, T x D;  z  device, T x D, or NULL (no gate)
 *   A         device, D x N, fp32;  D, dt_bias  device, D, fp32, or NULL
 *   B, C      device, T x G x N
 *   initial_state  device, S x D x N, fp32, or NULL (zeros)
 *   y         device, T x D
 *   final_state    device, S x D x N, fp32, or NULL
 *   workspace      device, 16-byte aligned, at least the bytes that
 *                  im2win_selective_scan_workspace_bytes gives (NULL when 0)
 * Errors: EINVAL, ENULL, EALIGN, EWORKSPACE, EOVERFLOW, EHIP.
 */
int im2win_selective_scan_workspace_bytes(const im2win_scan_desc* d, size_t* bytes);
int im2win_selective_scan(const im2win_scan_desc* d, const void* x, const void* dt, const float* A,
                          const void* B, const void* C, const float* D, const void* z,
                          const float* dt_bias, const int32_t* seq_starts, const float* initial_state,
                          void* y, float* final_state, void* workspace, size_t workspace_bytes,
                          void* stream);

/*
 * One token for each of d->tokens requests: the state of request i is
 * state[slots[i]] of a pool of state_slots states (D x N each, fp32), moved
 * on in place; slots as for im2win_causal_conv1d_step.
 * Errors: EINVAL, ENULL, EALIGN, EOVERFLOW, EHIP.
 */
int im2win_selective_scan_step(const im2win_scan_desc* d, const void* x, const void* dt, const float* A,
                               const void* B, const void* C, const float* D, const void* z,
                               const float* dt_bias, const int32_t* slots, float* state,
                               int64_t state_slots, void* y, void* stream);

/* Bytes of workspace that im2win_selective_scan_backward takes.  Host only. */
int im2win_selective_scan_backward_workspace_bytes(const im2win_scan_desc* d, size_t* bytes);

/*
 * Gradients of im2win_selective_scan for the gradient dy of y (T x D, dense)
 * and, where d_final_state (S x D x N, fp32) is given, of the final states.
 * The states are computed again; nothing of the forward call is needed.
 *   dx, ddt, dz   device, T x D (dz only where z is given, and then needed)
 *   dB, dC        device, T x G x N
 *   dA            device, D x N, fp32
 *   dD, ddt_bias  device, D, fp32, or NULL
 *   d_initial_state  device, S x D x N, fp32, or NULL
 *   workspace     device, 16-byte aligned, at least the bytes above
 * Errors: EINVAL, ENULL, EALIGN, EWORKSPACE, EOVERFLOW, EHIP.
 */
int im2win_selective_scan_backward(const im2win_scan_desc* d, const void* dy, const void* x, const void* dt,
                                   const float* A, const void* B, const void* C, const float* D,
                                   const void* z, const float* dt_bias, const int32_t* seq_starts,
                                   const float* initial_state, const float* d_final_state, void* dx,
                                   void* ddt, float* dA, void* dB, void* dC, float* dD, void* dz,
                                   float* ddt_bias, float* d_initial_state, void* workspace,
                                   size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------ */
/* Gated linear recurrence                                                   */
/* ------------------------------------------------------------------------ */

typedef struct {
    int64_t tokens;      /* T (requests, for the step) */
    int64_t channels;    /* D */
    int64_t sequences;   /* B >= 1 (not used by the step) */
    int64_t ld_x, ld_r, ld_i;    /* row strides of x, r and i */
    int32_t dtype;       /* of x, r, i, y and their gradients */
    float c;             /* > 0, the gate's exponent */
} im2win_recurrence_desc;

/*
 * For each channel, along each sequence, with s the logistic function,
 *   L[t] = -c softplus(lam) s(r[t]),  a[t] = exp(L[t]),
 *   h[t] = a[t] h[t-1] + sqrt(1 - a[t]^2) s(i[t]) x[t],   y[t] = h[t],
 * where the state before a sequence is its initial state, or zero.
 *   x, r, i  device, T x D
 *   lam      device, D, fp32
 *   initial_state  device, B x D, fp32, or NULL (zeros)
 *   y        device, T x D
 *   final_state    device, B x D, fp32, or NULL
 *   chunk_states   device, chunks x D, fp32, or NULL: the states that enter the
 *                  chunks of rows which the kernels work on, kept for the
 *                  gradients; im2win_gated_recurrence_chunks gives their number.
 *                  Where a sequence begins a chunk its row has no meaning.
 *   workspace      device, 16-byte aligned, at least the bytes that
 *                  im2win_gated_recurrence_workspace_bytes gives (NULL when 0)
 * Errors: EINVAL, ENULL, EALIGN, EWORKSPACE, EOVERFLOW, EHIP.
 */
int im2win_gated_recurrence_chunks(const im2win_recurrence_desc* d, int64_t* chunks);
int im2win_gated_recurrence_workspace_bytes(const im2win_recurrence_desc* d, size_t* bytes);
int im2win_gated_recurrence(const im2win_recurrence_desc* d, const void* x, const void* r, const void* i,
                            const float* lam, const int32_t* seq_starts, const float* initial_state,
                            void* y, float* final_state, float* chunk_states, void* workspace,
                            size_t workspace_bytes, void* stream);

/* Bytes of workspace that im2win_gated_recurrence_backward takes.  Host only. */
int im2win_gated_recurrence_backward_workspace_bytes(const im2win_recurrence_desc* d, size_t* bytes);

/*
 * Gradients of im2win_gated_recurrence for the gradient dy of y (T x D, dense)
 * and, where d_final_state (B x D, fp32) is given, of the final states.
 * chunk_states is what the forward call wrote for the same inputs, or NULL:
 * then it is computed again.
 *   dx, dr, di       device, T x D
 *   dlam             device, D, fp32
 *   d_initial_state  device, B x D, fp32, or NULL
 *   workspace        device, 16-byte aligned, at least the bytes above
 * Errors: EINVAL, ENULL, EALIGN, EWORKSPACE, EOVERFLOW, EHIP.
 */
int im2win_gated_recurrence_backward(const im2win_recurrence_desc* d, const void* dy, const void* x,
                                     const void* r, const void* i, const float* lam,
                                     const int32_t* seq_starts, const float* initial_state,
                                     const float* d_final_state, const float* chunk_states, void* dx,
                                     void* dr, void* di, float* dlam, float* d_initial_state,
                                     void* workspace, size_t workspace_bytes, void* stream);

/*
 * One token for each of d->tokens requests: the state of request i is
 * state[slots[i]] of a pool of state_slots states (D each, fp32), moved on in
 * place; slots as for im2win_causal_conv1d_step.
 * Errors: EINVAL, ENULL, EALIGN, EOVERFLOW, EHIP.
 */
int im2win_gated_recurrence_step(const im2win_recurrence_desc* d, const void* x, const void* r,
                                 const void* i, const float* lam, const int32_t* slots, float* state,
                                 int64_t state_slots, void* y, void* stream);

/* ------------------------------------------------------------------------ */
/* Norm of queries and keys for each head, with the position rotation        */
/* ------------------------------------------------------------------------ */

typedef struct {
    int64_t tokens;            /* T */
    int64_t q_heads, k_heads;  /* H and K heads a row, either may be 0 */
    int64_t head_dim;          /* channels of a head, even, 2 to 512 */
    int64_t rot_dim;           /* the first of them that are rotated, even, 0 to head_dim */
    int64_t ld_q, ld_k;        /* row strides of q and k */
    int32_t dtype;             /* of q, k, the outputs and their gradients */
    int32_t interleaved;       /* pairs (2p, 2p+1) where nonzero, (p, p + rot_dim/2) otherwise */
    float eps;                 /* >= 0 */
} im2win_qk_desc;

/*
 * For every head's channels x of a row t (w = wq or wk),
 *   u = x * rsqrt(mean(x^2) + eps) * w,
 *   (y[p], y[p']) = (u[p] cos - u[p'] sin, u[p'] cos + u[p] sin)
 * for the rotated pairs p, p' with the angle positions[t] * freqs[p] (radians);
 * y = u for the other channels.
 *   q, k       device, T x H x head_dim and T x K x head_dim, a row's heads
 *              one behind the other (a side without heads may be NULL)
 *   wq, wk     device, head_dim, fp32
 *   positions  device, T int32;  freqs  device, rot_dim/2, fp32 (both may be
 *              NULL where rot_dim is 0)
 *   yq, yk     device, dense; yq may be q itself where q is dense, yk likewise
 * Errors: EINVAL, ENULL, EALIGN, EOVERFLOW, EHIP.
 */
int im2win_qk_norm_rope(const im2win_qk_desc* d, const void* q, const void* k, const float* wq,
                        const float* wk, const int32_t* positions, const float* freqs, void* yq,
                        void* yk, void* stream);

/* Bytes of workspace that im2win_qk_norm_rope_backward takes.  Host only. */
int im2win_qk_norm_rope_backward_workspace_bytes(const im2win_qk_desc* d, size_t* bytes);

/*
 * Gradients for dyq and dyk (dense), with the q and k that the forward call read.
 *   dq, dk    device, dense; dq may be dyq itself, dk likewise
 *   dwq, dwk  device, head_dim, fp32 (zeros for a side without heads)
 *   workspace device, 16-byte aligned, at least the bytes above
 * Errors: EINVAL, ENULL, EALIGN, EWORKSPACE, EOVERFLOW, EHIP.
 */
int im2win_qk_norm_rope_backward(const im2win_qk_desc* d, const void* dyq, const void* dyk, const void* q,
                                 const void* k, const float* wq, const float* wk,
                                 const int32_t* positions, const float* freqs, void* dq, void* dk,
                                 float* dwq, float* dwk, void* workspace, size_t workspace_bytes,
                                 void* stream);

/* ------------------------------------------------------------------------ */
/* Attention with a sliding window and first tokens that stay visible        */
/* ------------------------------------------------------------------------ */

typedef struct {
    int64_t tokens;            /* T, at most 2^29 (requests, for the step) */
    int64_t sequences;         /* B >= 1 (not used by the step) */
    int64_t q_heads, kv_heads; /* H and K; query head h reads key head h / (H / K) */
    int64_t head_dim;          /* a multiple of 8 up to 256 */
    int64_t window;            /* W, 1 to 2^30: a token sees itself and the W-1 before it */
    int64_t sinks;             /* S, 0 to 32: and the first S of its sequence */
    int64_t ld_q, ld_k, ld_v;  /* row strides of q, k and v, below 2^24 */
    int32_t dtype;             /* of q, k, v, the caches, y and the gradients */
    float scale;               /* > 0 */
} im2win_window_desc;

/*
 * y[t][h] = sum_j w[j] v[j], w = softmax over j of scale * q[t][h] . k[j], for
 * the positions j <= p of t's sequence with j > p - W or j < S, where p is
 * t's position: past[b] + its row in the sequence.  Positions below past[b]
 * are read from the request's cache, the others are the call's own rows.  A
 * masked position does not enter, whatever its key and value hold.
 *   q, k, v  device, T x H x head_dim and T x K x head_dim (k, v)
 *   k_cache, v_cache  device, cache_slots x (S + W) x K x head_dim, or both
 *            NULL: position j lies in row j where j < S, else in row
 *            S + (j - S) mod W.  The call reads what lies before past[b] and
 *            leaves the new tokens' keys and values there.
 *   past     device, B int32, or NULL (zeros): tokens that the request had
 *            before the call; values outside of [0, 2^30] are taken as the nearest
 *   slots    device, B int32, or NULL (b): the request's slot of the cache.  No
 *            two requests may name the same slot.  A request whose slot is
 *            outside of [0, cache_slots) gets y = 0 and leaves the cache as it is.
 *   y        device, T x H x head_dim
 *   lse      device, T x H, fp32, or NULL: log of the sum of exp(scale q . k) (-inf
 *            for a request without a slot), for the gradients
 * Where all of a query's scores are -inf, y is NaN and lse -inf, as the formula has it.
 * Errors: EINVAL, ENULL, EALIGN, EOVERFLOW, EHIP.
 */
int im2win_window_attention(const im2win_window_desc* d, const void* q, const void* k, const void* v,
                            const int32_t* seq_starts, void* k_cache, void* v_cache,
                            int64_t cache_slots, const int32_t* past, const int32_t* slots, void* y,
                            float* lse, void* stream);

/* Bytes of workspace that im2win_window_attention_step takes.  Host only. */
int im2win_window_attention_step_workspace_bytes(const im2win_window_desc* d, size_t* bytes);

/*
 * One token for each of d->tokens requests, at position past[i]: its key and
 * value (rows of k and v) go to the request's cache, and y is the attention
 * over what the cache then holds of the request.  past is needed and is not
 * moved on; cache and slots as above.
 *   workspace  device, 16-byte aligned, at least the bytes above (NULL when 0)
 * Errors: EINVAL, ENULL, EALIGN, EWORKSPACE, EOVERFLOW, EHIP.
 */
int im2win_window_attention_step(const im2win_window_desc* d, const void* q, const void* k,
                                 const void* v, void* k_cache, void* v_cache, int64_t cache_slots,
                                 const int32_t* past, const int32_t* slots, void* y, void* workspace,
                                 size_t workspace_bytes, void* stream);

/* Bytes of workspace that im2win_window_attention_backward takes.  Host only. */
int im2win_window_attention_backward_workspace_bytes(const im2win_window_desc* d, size_t* bytes);

/*
 * Gradients of im2win_window_attention without a cache, for dy (dense), with
 * the y and lse that the forward call wrote.  A masked pair does not enter:
 * an infinity or a NaN reaches what the formulas over the pairs in sight give it.
 *   dq          device, T x H x head_dim, dense
 *   dk, dv      device, T x K x head_dim, dense
 *   workspace   device, 16-byte aligned, at least the bytes above
 * Errors: EINVAL, ENULL, EALIGN, EWORKSPACE, EOVERFLOW, EHIP.
 */
int im2win_window_attention_backward(const im2win_window_desc* d, const void* dy, const void* q,
                                     const void* k, const void* v, const void* y, const float* lse,
                                     const int32_t* seq_starts, void* dq, void* dk, void* dv,
                                     void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* IM2WIN_SEQ_H */
