/*
 * im2win_seq.h -- operators over sequences of tokens: the short causal
 * convolution of state space layers (a depthwise convolution along time),
 * the selective state space scan that reads its output, and the
 * root-mean-square norm with the residual's addition in front of both.
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

#ifdef __cplusplus
}
#endif

#endif /* IM2WIN_SEQ_H */
