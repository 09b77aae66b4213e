// Gradients of window attention.  With the weights w = exp(scale q k - lse) of
// the forward call, dp = dy v and delta = dy y (over the channels),
//   ds = w (dp - delta),  dq = scale sum_j ds k_j,
//   dk = scale sum_t ds q_t,  dv = sum_t w dy_t.
// A query that sees one key alone has w = 1 whatever its score: its ds is zero,
// and taken as such where it is finite.
//
// Three kernels, none of which stores scores or adds atomically:
//  - queries' tiles walk their visible keys (dq, and delta for the others);
//  - keys' tiles walk the queries of all their heads that see them by the
//    window (dk, dv);
//  - the first tokens' keys are seen by all queries behind: those pairs, cut
//    into pieces of queries, leave partial sums, which the tile of the
//    sequence's first keys adds (launched before it).
// The matrix products multiply an infinity or a NaN in a masked place by zero:
// where results are not finite, a wave computes them again from the pairs in
// sight alone.
// Scores are computed twice: seven products of queries and keys where five
// would do (ten in bf16, where weights and ds have two parts), against a sum of
// dq over the keys' tiles in memory.
//
// 16384 tokens of 16 heads over 4, 128 bf16 channels, window 1024, 4 first
// tokens: 291 us for dq, 45 for the first tokens' keys, 480 for dk and dv; the
// products of all pairs in sight, at the rate of a large one, would take 215, 1
// and 322.  The operands' way out of LDS and the exponentials take the rest:
// matrix cores are busy for 43% and 38% of the time of dq and of dk and dv, and
// waves wait for 38% and 56% of theirs.  2503 tokens of 6 heads over 2, 96 fp32
// channels, window 201: 52, 31 and 60 us, latency of few workgroups.
#include "seq_attention.h"

#include <algorithm>

namespace im2win {
namespace {

struct AttnBwdArgs {
    const void *dy, *q, *k, *v, *y;
    const float* lse;
    void *dq, *dk, *dv;
    float *delta, *part;           // part: place x key head x (dk, dv) x sinks x channels
    SeqMap seq;
    int64_t ld_q, ld_k, ld_v;
    int64_t q_places, q_items, k_places, k_items, pieces;
    int q_heads, kv_heads, dim, window, sinks;
    int pack, tile, piece;         // piece: queries whose sums for the first tokens' keys go together
    float c, scale;
};

template <typename T>
__device__ __forceinline__ Frag<T> load_frag(const T* row, int s, int half, int dim) {
    Frag<T> f;
    if (16 * s + 8 * half < dim) f.load(row + 16 * s + 8 * half);
    else f.zero();
    return f;
}

// Rows of the keys' kernel's tiles of queries: of 128 bf16 channels 32 (a training
// step of 16384 tokens with a window of 16: 235 us, 251 with 64; of 1024 1067 with
// both).  The queries' kernel's tiles of keys are of 64 rows there (1067 us, 1081
// with 32).
template <typename T, int DP> constexpr int kTileRows = sizeof(T) == 2 && DP <= 96 ? 64 : 32;
// Queries that see fewer keys than this walk them twice: all of them with windows
// below it, otherwise the first workgroups of each sequence.  Without the
// correction, the error of dq is 1.95 times its own rounding's where two keys are
// seen, 1.25 where eight are, 1.10 where 24 are and under 1.06 from 64 on.  It costs
// the walk's scores again: a training step of 16384 tokens of 16 x 128 with a window
// of 16 226 -> 235 us, of 16 key heads of 64 with one of 48 194 -> 209.
constexpr int kFewKeys = 64;
// Waves a SIMD, of dq by its registers (training steps: 16384 tokens of 16 x 64 bf16
// 573 us with three waves, 578 with two; 8192 tokens of 16 heads of 96 fp32 1100 with
// two, 1153 with one, of 128 fp32 1468 and 1538; of 192 bf16 557 with two, 561 with
// one), of dk and dv fewer, which hold the sums of both (16 x 128 bf16 1067 with two,
// 1173 with one; 16 x 64 bf16 569 with two, 623 with three; 96 fp32 1100 with one,
// 1342 with two, 128 fp32 1468 and 1940; 192 bf16 561 and 1161).
template <typename T, int DP> constexpr int kDqWaves = DP > 128 ? 1 : sizeof(T) == 2 && DP <= 64 ? 3 : 2;
template <typename T, int DP> constexpr int kDkvWaves = DP * sizeof(T) > 256 ? 1 : 2;

// ---------------------------------------------------------------------------
// Results that are not finite, from the formulas over the pairs in sight: for the
// few places that stand in a block with an infinity or a NaN that they do not see.
// A wave takes a query, or a key: its lanes compute 64 pairs' weights and ds, a
// pair each, and then add the pairs' rows one after the other, a channel each.
// Where lse or delta is not finite itself, all results are NaN already.
// ---------------------------------------------------------------------------
constexpr int kLaneChannels = 4;       // 256 channels

// Channels lane, lane + 64, .. of a row
template <typename T>
struct Row {
    float v[kLaneChannels] = {};
    __device__ __forceinline__ Row() {}
    __device__ __forceinline__ Row(const T* p, int lane, int dim) {
#pragma unroll
        for (int i = 0; i < kLaneChannels; ++i) {      // (loads of all lanes, which can be under way together)
            const T x = p[lane + i * kWave < dim ? lane + i * kWave : 0];
            v[i] = lane + i * kWave < dim ? (float)x : 0.0f;
        }
    }
    __device__ __forceinline__ void add(float w, const Row& o) {
#pragma unroll
        for (int i = 0; i < kLaneChannels; ++i) v[i] = fmaf(w, o.v[i], v[i]);
    }
    __device__ __forceinline__ void put(T* p, int lane, int dim, float scale) const {
#pragma unroll
        for (int i = 0; i < kLaneChannels; ++i)
            if (lane + i * kWave < dim) p[lane + i * kWave] = (T)(v[i] * scale);
    }
};

// The product of a lane's rows
template <typename T>
__device__ __forceinline__ float dot(const T* a, const T* b, int dim) {
    float s = 0.0f;
    for (int c = 0; c < dim; c += 8) {
        Frag<T> x, y;
        x.load(a + c);
        y.load(b + c);
#pragma unroll
        for (int i = 0; i < 8; ++i) s = fmaf(x.get(i), y.get(i), s);
    }
    return s;
}

template <typename T>
__device__ __forceinline__ void repair_query(const AttnBwdArgs& a, const SeqTile& st, int pos, int head, float delta) {
    const int lane = threadIdx.x % kWave, kvh = head / (a.q_heads / a.kv_heads);
    const int64_t t = st.first + pos, at = t * a.q_heads + head;
    const float lse = a.lse[at] * kLog2e;
    if (!__ballot(finite(lse) && finite(delta))) return;
    const T *q = static_cast<const T*>(a.q) + t * a.ld_q + (int64_t)head * a.dim, *g = static_cast<const T*>(a.dy) + at * a.dim;
    const int low = pos - a.window + 1 > 0 ? pos - a.window + 1 : 0, first = a.sinks < low ? a.sinks : low, count = first + pos + 1 - low;
    const float several = pos == 0 || (a.window == 1 && a.sinks == 0) ? 0.0f : 1.0f;
    auto key = [&](int n) { return (int64_t)st.first + (n < first ? n : low + n - first); };
    Row<T> sum;
    for (int n0 = 0; n0 < count; n0 += kWave) {
        const int here = count - n0 < kWave ? count - n0 : kWave;
        const int64_t mine = key(n0 + (lane < here ? lane : 0));
        const float s = dot(static_cast<const T*>(a.k) + mine * a.ld_k + (int64_t)kvh * a.dim, q, a.dim), dp = dot(static_cast<const T*>(a.v) + mine * a.ld_v + (int64_t)kvh * a.dim, g, a.dim);
        const float ds = __builtin_amdgcn_exp2f(fmaf(s, a.c, -lse)) * (dp - delta) * several;
#pragma unroll 8
        for (int r = 0; r < here; ++r) sum.add(__shfl(ds, r), Row<T>(static_cast<const T*>(a.k) + key(n0 + r) * a.ld_k + (int64_t)kvh * a.dim, lane, a.dim));
    }
    sum.put(static_cast<T*>(a.dq) + at * a.dim, lane, a.dim, a.scale);
}

template <typename T>
__device__ __forceinline__ void repair_key(const AttnBwdArgs& a, const SeqTile& st, int key, int kvh, bool need_k, bool need_v) {
    const int lane = threadIdx.x % kWave, group = a.q_heads / a.kv_heads;
    const int64_t t = st.first + key, to = (t * a.kv_heads + kvh) * a.dim;
    T *dk = static_cast<T*>(a.dk) + to, *dv = static_cast<T*>(a.dv) + to;
    const int end = key < a.sinks || st.len - key < a.window ? st.len : key + a.window;
    auto row = [&](int p, int h) { return (int64_t)(st.first + p) * a.q_heads + kvh * group + h; };
    // What the rows in sight account for: dk where a delta is not finite, and the
    // channels of dv where that row's dy (whose every infinity shows in delta) is not.
    Row<T> open(dv, lane, a.dim);
    for (int h = 0; h < group; ++h)
        for (int p0 = key; p0 < end; p0 += kWave) {
            const int64_t mine = row(p0 + lane < end ? p0 + lane : end - 1, h);
            if (__ballot(!finite(a.lse[mine]))) return;
            uint64_t bad = __ballot(p0 + lane < end && !finite(a.delta[mine]));
            if (bad) need_k = false;
            for (; bad && need_v; bad &= bad - 1) {
                const Row<T> g(static_cast<const T*>(a.dy) + row(p0 + __builtin_ctzll(bad), h) * a.dim, lane, a.dim);
                bool any = false;
#pragma unroll
                for (int i = 0; i < kLaneChannels; ++i) {
                    open.v[i] = finite(g.v[i]) ? open.v[i] : 0.0f;
                    any |= !finite(open.v[i]);
                }
                need_v = __ballot(any);
            }
            if (!need_k && !need_v) return;
        }
    const T *k = static_cast<const T*>(a.k) + t * a.ld_k + (int64_t)kvh * a.dim, *v = static_cast<const T*>(a.v) + t * a.ld_v + (int64_t)kvh * a.dim;
    Row<T> sum_k, sum_v;
    for (int h = 0; h < group; ++h)
        for (int p0 = key; p0 < end; p0 += kWave) {
            const int here = end - p0 < kWave ? end - p0 : kWave, mine = p0 + (lane < here ? lane : 0);
            auto query = [&](int p) { return static_cast<const T*>(a.q) + (int64_t)(st.first + p) * a.ld_q + (int64_t)(kvh * group + h) * a.dim; };
            auto grad = [&](int p) { return static_cast<const T*>(a.dy) + row(p, h) * a.dim; };
            const float w = __builtin_amdgcn_exp2f(fmaf(dot(query(mine), k, a.dim), a.c, -a.lse[row(mine, h)] * kLog2e));
            const float ds = w * (dot(grad(mine), v, a.dim) - a.delta[row(mine, h)]) * (mine == 0 || (a.window == 1 && a.sinks == 0) ? 0.0f : 1.0f);
#pragma unroll 8
            for (int r = 0; r < here; ++r) {
                sum_v.add(__shfl(w, r), Row<T>(grad(p0 + r), lane, a.dim));
                sum_k.add(__shfl(ds, r), Row<T>(query(p0 + r), lane, a.dim));
            }
        }
    if (need_k) sum_k.put(dk, lane, a.dim, a.scale);
    if (need_v) sum_v.put(dv, lane, a.dim, 1.0f);
}

// The kernel's arguments (it has no others), loaded again, and its block: what the
// second computation needs is worked out anew, since held over the walk it would
// take the walk's registers (a training step of 16384 tokens 925 us, 903 so).
struct Again : AttnBwdArgs {
    int block;
};
__device__ __forceinline__ Again arguments() {
    typedef const __attribute__((address_space(4))) uint64_t* Words;
    Words p = (Words)__builtin_amdgcn_kernarg_segment_ptr();
    int block = blockIdx.x;
    asm volatile("" : "+s"(p), "+s"(block));
    constexpr int N = sizeof(AttnBwdArgs) / 8;
    static_assert(sizeof(AttnBwdArgs) % 8 == 0, "whole words");
    uint64_t w[N];
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = p[i];
    Again a;
    __builtin_memcpy(static_cast<AttnBwdArgs*>(&a), w, sizeof(AttnBwdArgs));
    a.block = block;
    return a;
}

// The queries (columns of the wave) of a tile, and keys (from `from` on), with a bit each
template <typename T>
__device__ __forceinline__ void repair_queries(uint32_t bad, float delta) {
    const Again a = arguments();
    const int64_t item = die_order(a.block, a.q_items);
    const SeqTile st = seq_tile(a.seq, (int)(item % a.q_places), a.tile);
    for (; bad; bad &= bad - 1) {
        const int c = __builtin_ctz(bad), n = uniform(threadIdx.x / kWave) * kCols + c;
        repair_query<T>(a, st, st.row + n / a.pack, (int)(item / a.q_places) * a.pack + n % a.pack, __shfl(delta, c));
    }
}
template <typename T>
__device__ __forceinline__ void repair_keys(const AttnBwdArgs& a, const SeqTile& st, int kvh, int from, uint32_t bad_k, uint32_t bad_v) {
    for (uint32_t bad = uniform(bad_k | bad_v); bad; bad &= bad - 1) {
        const int c = __builtin_ctz(bad);
        repair_key<T>(a, st, st.row + uniform(from) + c, kvh, bad_k >> c & 1, bad_v >> c & 1);
    }
}
// (Called where the walk spills by the hundreds: 4096 tokens of 8 x 256 fp32 1541 us
// with it inlined, 1433 so; narrower walks have registers that a call would take.)
template <typename T>
__device__ __attribute__((noinline)) void call_repair_keys(const AttnBwdArgs& a, const SeqTile& st, int kvh, int from, uint32_t bad_k, uint32_t bad_v) {
    repair_keys<T>(a, st, kvh, from, bad_k, bad_v);
}
template <typename T, int DP>
__device__ __forceinline__ void repair_tile(const AttnBwdArgs& a, const SeqTile& st, int kvh, int from, uint32_t bad_k, uint32_t bad_v) {
    if constexpr (DP * sizeof(T) > 768) call_repair_keys<T>(a, st, kvh, from, bad_k, bad_v);
    else repair_keys<T>(a, st, kvh, from, bad_k, bad_v);
}

// ---------------------------------------------------------------------------
// dq and delta: workgroups and columns as in the forward kernel
// ---------------------------------------------------------------------------
template <typename T, int DP>
__global__ __launch_bounds__(kAttnThreads, (kDqWaves<T, DP>)) void window_dq_kernel(AttnBwdArgs a) {
    constexpr int BK = sizeof(T) == 2 && DP <= 128 ? 64 : 32, NB = BK / 32;
    using KV = Tile<T, DP, BK>;
    using Copy = Feed<T, DP, BK>;
    constexpr int kAhead = kAheadTiles<KV::kBytes, kDqWaves<T, DP>>, kBuffers = kAhead + 1;
    __shared__ __align__(128) char lds[2 * kBuffers * KV::kBytes];      // buffers of keys, then of values
    const int64_t item = die_order(blockIdx.x, a.q_items);
    if (item >= a.q_items) return;
    const int hb = (int)(item / a.q_places);
    const SeqTile st = seq_tile(a.seq, (int)(item % a.q_places), a.tile);
    if (st.row >= st.len) return;
    const int tid = threadIdx.x, wave = uniform(tid / kWave), lane = tid % kWave, half = lane / 32;
    const int h0 = hb * a.pack, kvh = h0 / (a.q_heads / a.kv_heads);
    const int col = wave * kCols + lane % kCols, qi = col / a.pack, row = st.row + qi;
    const bool live = qi < a.tile && row < st.len;
    const int last = st.row + a.tile < st.len ? st.row + a.tile - 1 : st.len - 1;
    const int pos = row < last ? row : last, head = h0 + col % a.pack;
    const int64_t t = st.first + pos, at = t * a.q_heads + head;
    Frag<T> q[DP / 16], g[DP / 16];
    float delta = 0.0f;
    const T* qp = static_cast<const T*>(a.q) + t * a.ld_q + (int64_t)head * a.dim;
#pragma unroll
    for (int s = 0; s < DP / 16; ++s) {
        q[s] = load_frag(qp, s, half, a.dim);
        g[s] = load_frag(static_cast<const T*>(a.dy) + at * a.dim, s, half, a.dim);
        const Frag<T> y = load_frag(static_cast<const T*>(a.y) + at * a.dim, s, half, a.dim);
#pragma unroll
        for (int i = 0; i < 8; ++i) delta = fmaf(g[s].get(i), y.get(i), delta);
    }
    delta = half_sum(delta);
    const float lse = a.lse[at] * kLog2e;
    const float several = pos == 0 || (a.window == 1 && a.sinks == 0) ? 0.0f : 1.0f;      // keys seen

    const int begin = st.row - a.window + 1 > 0 ? st.row - a.window + 1 : 0;
    const int first_end = a.sinks < begin ? a.sinks : begin, end = last + 1;
    const int wq0 = st.row + wave * kCols / a.pack;
    int wq1 = st.row + (wave * kCols + kCols - 1) / a.pack;
    wq1 = wq1 < last ? wq1 : last;
    const Copy ck(a.ld_k), cv(a.ld_v);
    const char* kp = reinterpret_cast<const char*>(static_cast<const T*>(a.k) + st.first * a.ld_k + (int64_t)kvh * a.dim);
    const char* vp = reinterpret_cast<const char*>(static_cast<const T*>(a.v) + st.first * a.ld_v + (int64_t)kvh * a.dim);
    auto issue = [&](int buffer, int base, int stop) {
        ck.issue(lds + buffer * KV::kBytes, kp + (int64_t)base * ck.stride, stop - base, a.dim);
        cv.issue(lds + (kBuffers + buffer) * KV::kBytes, vp + (int64_t)base * cv.stride, stop - base, a.dim);
    };
    const int rb = KV::row_base(lane), cb = KV::col_base(lane);
    f32x16 o[DP / 32];
#pragma unroll
    for (int i = 0; i < DP / 32; ++i) o[i] = f32x16{};
    if (a.dim != DP) clear(lds, 2 * kBuffers * KV::kBytes);
    // tile i: the sinks', where there is one, and those of the windows
    const int lead = first_end > 0 ? 1 : 0, count = lead + (end - begin + BK - 1) / BK;
    auto base_of = [&](int i) { return i < lead ? 0 : begin + (i - lead) * BK; };
    auto stop_of = [&](int i) { return i < lead ? first_end : end; };
    // delta comes from the y that was rounded, which shows where few keys are
    // seen: there a first walk finds what ds sums to over the keys, zero but for
    // delta's error, and corrects it
    float rest = 0.0f;
    const bool few = st.row + 1 < kFewKeys || a.window + a.sinks < kFewKeys;      // keys of the tile's first query
    for (int walk = sizeof(T) == 2 && few ? 0 : 1; walk < 2; ++walk) {
        for (int i = 0; i < kAhead && i < count; ++i) issue(i, base_of(i), stop_of(i));
        int buffer = 0;
        for (int n = 0; n < count; ++n) {
            const bool sink_tile = n < lead;
            const int now = base_of(n), now_stop = stop_of(n), newest = n + kAhead - 1;
            arrived<2 * Copy::kPasses>(kAhead == 2 && newest < count && a.dim == DP && base_of(newest) + BK <= stop_of(newest));
            const int before = buffer ? buffer - 1 : kBuffers - 1;
            if (n + kAhead < count) issue(before, base_of(n + kAhead), stop_of(n + kAhead));
            const int kb = rb + buffer * KV::kBytes, kc = cb + buffer * KV::kBytes, vb = rb + (kBuffers + buffer) * KV::kBytes;
            buffer = buffer + 1 < kBuffers ? buffer + 1 : 0;
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                // 32 keys that all of the wave's queries see, or none (taken tile by
                // tile instead, a training step of 16384 tokens took 937 us, not 908)
                const int from = now + 32 * b;
                if (from > wq1 || (from + 32 <= wq0 - a.window + 1 && from >= a.sinks) || (b && sink_tile)) continue;
                const bool whole = !sink_tile && from >= a.sinks && from + 31 <= wq0 && from > wq1 - a.window;
                f32x16 s = {}, dp = {};
#pragma unroll
                for (int d = 0; d < DP / 16; ++d) {
                    mma(s, KV::row_frag(lds, kb, b, d), q[d]);
                    mma(dp, KV::row_frag(lds, vb, b, d), g[d]);
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], a.c, -lse)) * (dp[i] - delta);
                if (!whole) {
                    const int low = pos - a.window + 1 - now - 4 * half, high = now_stop - now - 4 * half;
                    if (sink_tile) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) s[i] = 32 * b + acc_row(i, 0) < high ? s[i] : 0.0f;
                    } else if (now >= a.sinks) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) s[i] = (uint32_t)(32 * b + acc_row(i, 0) - low) < (uint32_t)a.window ? s[i] * several : 0.0f;
                    } else {
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const int p = now + 32 * b + acc_row(i, half);
                            s[i] = p <= pos && (p > pos - a.window || p < a.sinks) ? s[i] * several : 0.0f;
                        }
                    }
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) rest += s[i];
                if (walk == 0) continue;
#pragma unroll
                for (int part = 0; part < 2; ++part) {
                    const Parts<T> w(s, part);
#pragma unroll
                    for (int d = 0; d < DP / 32; ++d) mma(o[d], KV::col_frag(lds, kc, d, 2 * b + part), w);
                }
            }
        }
        if (walk == 0) {
            delta += half_sum(rest);
            rest = 0.0f;
            __syncthreads();
        }
    }
    // ds sums to zero over the keys: what it sums to is what delta is off by, from the rounded y
    rest = half_sum(rest);
    delta += rest;
    if (live && half == 0) a.delta[at] = delta;
    T* dq = static_cast<T*>(a.dq) + at * a.dim;
    const uint64_t bad = __ballot(live && nonfinite(o));
#pragma unroll
    for (int b = 0; b < DP / 32; ++b)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const int d = 32 * b + acc_row(i, half);
            if (live && d < a.dim) put4(dq + d, o[b][i] * a.scale, o[b][i + 1] * a.scale, o[b][i + 2] * a.scale, o[b][i + 3] * a.scale);
        }
    if (bad) repair_queries<T>((uint32_t)bad | (uint32_t)(bad >> 32), delta);
}

// ---------------------------------------------------------------------------
// A block of 32 queries in LDS against the wave's 32 keys, one a lane's
// column: w and ds stay in the accumulators and are the right operands of
// dv^T += dy^T w and dk^T += q^T ds.
// ---------------------------------------------------------------------------
template <typename T, int DP>
struct Keys {
    Frag<T> k[DP / 16], v[DP / 16];
    f32x16 dk[DP / 32], dv[DP / 32];
    int rb, cb;                  // the lane's places in a tile

    __device__ __forceinline__ void load(const T* kp, const T* vp, int half, int dim, bool live) {
#pragma unroll
        for (int s = 0; s < DP / 16; ++s) {
            if (live) {
                k[s] = load_frag(kp, s, half, dim);
                v[s] = load_frag(vp, s, half, dim);
            } else {
                k[s].zero();
                v[s].zero();
            }
        }
#pragma unroll
        for (int d = 0; d < DP / 32; ++d) dk[d] = dv[d] = f32x16{};
        rb = Tile<T, DP, 32>::row_base(threadIdx.x % kWave);
        cb = Tile<T, DP, 32>::col_base(threadIdx.x % kWave);
    }
    // seen(position) for the lane's key, and single(position), where the block
    // is not seen as a whole; qt and gt are the tiles' places in LDS, lse and delta
    // their rows' there.
    template <int R, typename F, typename G>
    __device__ __forceinline__ void take(const char* lds, int qt, int gt, const float* lse, const float* delta, int b, int base, bool whole, float c, F seen, G single) {
        using Q = Tile<T, DP, R>;
        const int lane = threadIdx.x % kWave, half = lane / 32;
        f32x16 s = {}, dp = {};
#pragma unroll
        for (int d = 0; d < DP / 16; ++d) {
            mma(s, Q::row_frag(lds, rb + qt, b, d), k[d]);
            mma(dp, Q::row_frag(lds, rb + gt, b, d), v[d]);
        }
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            float l[4], e[4];
            __builtin_memcpy(l, lse + 32 * b + acc_row(i, half), 16);
            __builtin_memcpy(e, delta + 32 * b + acc_row(i, half), 16);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                s[i + j] = __builtin_amdgcn_exp2f(fmaf(s[i + j], c, -l[j]));
                dp[i + j] = s[i + j] * (dp[i + j] - e[j]);
            }
        }
        if (!whole) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int p = base + 32 * b + acc_row(i, half);
                const bool in = seen(p);
                s[i] = in ? s[i] : 0.0f;
                dp[i] = in ? dp[i] * (single(p) ? 0.0f : 1.0f) : 0.0f;
            }
        }
#pragma unroll
        for (int part = 0; part < 2; ++part) {
            const Weights<T> w(s, part);
            const Parts<T> ds(dp, part);
            __builtin_amdgcn_s_setprio(1);      // products first; keeps the exponentials in front of them (8192 tokens of 16 x 32 fp32: 454 -> 445 us)
#pragma unroll
            for (int d = 0; d < DP / 32; ++d) {
                mma(dv[d], Q::col_frag(lds, cb + gt, d, 2 * b + part), w);
                mma(dk[d], Q::col_frag(lds, cb + qt, d, 2 * b + part), ds);
            }
            __builtin_amdgcn_s_setprio(0);
        }
    }
};

// Pieces of the sequences that are longer than the window, of which tokens / (window
// + 1) can exist, whatever the number of sequences: where seq_starts is given,
// sequence b, from row f on, owns the places from f / piece + min(b, f / (window + 1))
// on.  Behind a sequence that is longer that is larger by its pieces at least;
// behind others it may not be, and the last of those that begin at a place has it.
__device__ __forceinline__ int first_piece(const AttnBwdArgs& a, int b, int first) {
    const int longer = first / (a.window + 1);
    return first / a.piece + (b < longer ? b : longer);
}
__device__ __forceinline__ SeqTile piece_tile(const AttnBwdArgs& a, int place) {
    if (!a.seq.starts) return seq_tile(a.seq, place, a.piece);
    return find_tile(a.seq, place, a.piece, [&](int b) { return first_piece(a, b, a.seq.clamped(b)); });
}

// The sums that the first tokens' pieces of a sequence left, for the tile of its first keys
struct FirstSums {
    bool any;
    int pieces;
    int64_t count, step;      // values of a piece, from one piece to the next
    float* part;
    __device__ __forceinline__ FirstSums(const AttnBwdArgs& a, const SeqTile& st, int kvh) {
        any = a.sinks && st.len > a.window;
        const int from = a.window / a.piece, place = a.seq.starts ? first_piece(a, st.b, st.first) : st.b * ((a.seq.len + a.piece - 1) / a.piece);
        pieces = (st.len + a.piece - 1) / a.piece - from;
        count = 2 * (int64_t)a.sinks * a.dim;
        step = a.kv_heads * count;
        part = a.part + ((int64_t)(place + from) * a.kv_heads + kvh) * count;
    }
    // All of them into the first piece's: by all threads of the workgroup, in front of a barrier
    __device__ __forceinline__ void add(int tid, int threads) const {
        if (pieces < 2) return;
        for (int n = tid; n < count; n += threads) {
            float v = 0.0f;
#pragma unroll 8
            for (int z = 0; z < pieces; ++z) v += part[z * step + n];
            part[n] = v;
        }
    }
};

template <typename T, int DP>
__global__ __launch_bounds__(kAttnThreads, (kDkvWaves<T, DP>)) void window_dkv_kernel(AttnBwdArgs a) {
    constexpr int BQ = kTileRows<T, DP>, NB = BQ / 32;
    using Q = Tile<T, DP, BQ>;
    using Copy = Feed<T, DP, BQ>;
    constexpr int kAhead = kAheadTiles<Q::kBytes, kDkvWaves<T, DP>>, kBuffers = kAhead + 1;
    __shared__ __align__(128) char lds[2 * kBuffers * Q::kBytes];      // buffers of queries, then of gradients
    __shared__ __align__(16) float lse[kBuffers][BQ], delta[kBuffers][BQ];
    const int64_t item = die_order(blockIdx.x, a.k_items);
    if (item >= a.k_items) return;
    const int kvh = (int)(item / a.k_places);
    const SeqTile st = seq_tile(a.seq, (int)(item % a.k_places), kGroupCols);
    if (st.row >= st.len) return;
    const int tid = threadIdx.x, wave = uniform(tid / kWave), lane = tid % kWave, half = lane / 32;
    const int group = a.q_heads / a.kv_heads;
    const int key = st.row + wave * kCols + lane % kCols;      // the lane's column
    const bool live = key < st.len;
    const int k0 = st.row + wave * kCols, k1 = k0 + kCols - 1;
    Keys<T, DP> keys;
    keys.load(static_cast<const T*>(a.k) + (int64_t)(st.first + key) * a.ld_k + (int64_t)kvh * a.dim,
              static_cast<const T*>(a.v) + (int64_t)(st.first + key) * a.ld_v + (int64_t)kvh * a.dim, half, a.dim, live);

    // queries that see some key of the tile by the window
    const int begin = st.row, far = st.row + kGroupCols - 1 + a.window;
    const int end = far < st.len ? far : st.len;
    const Copy cq(a.ld_q), cg((int64_t)a.q_heads * a.dim);
    const char* qp = reinterpret_cast<const char*>(static_cast<const T*>(a.q) + st.first * a.ld_q + (int64_t)kvh * group * a.dim);
    const char* gp = reinterpret_cast<const char*>(static_cast<const T*>(a.dy) + ((int64_t)st.first * a.q_heads + kvh * group) * a.dim);
    float lr = 0.0f, er = 0.0f;
    auto issue = [&](int buffer, int g, int base) {
        if (tid < BQ) {
            const int64_t at = (int64_t)(st.first + base + tid) * a.q_heads + kvh * group + g;
            lr = base + tid < end ? a.lse[at] * kLog2e : 0.0f;
            er = base + tid < end ? a.delta[at] : 0.0f;
        }
        const int64_t head = (int64_t)g * a.dim * (int)sizeof(T);
        cq.issue(lds + buffer * Q::kBytes, qp + head + (int64_t)base * cq.stride, end - base, a.dim);
        cg.issue(lds + (kBuffers + buffer) * Q::kBytes, gp + head + (int64_t)base * cg.stride, end - base, a.dim);
    };
    const FirstSums first(a, st, kvh);
    const bool first_keys = st.row == 0 && first.any;
    if (first_keys) first.add(tid, kAttnThreads);
    // tiles of queries, one head after the other; lse and delta of a tile wait
    // in registers from its issue to the next iteration
    if (a.dim != DP) clear(lds, 2 * kBuffers * Q::kBytes);
    const int count = group * ((end - begin + BQ - 1) / BQ);
    int ahead_g = 0, ahead_base = begin, ahead = 0, held = -1, buffer = 0, now = begin;
    bool newest_whole = false;
    auto advance = [&](int& g, int& b) {
        b += BQ;
        if (b >= end) b = begin, ++g;
    };
    auto keep = [&] {
        if (held >= 0 && tid < BQ) lse[held][tid] = lr, delta[held][tid] = er;
    };
    auto next = [&](int into) {
        issue(into, ahead_g, ahead_base);
        newest_whole = a.dim == DP && ahead_base + BQ <= end;
        held = into;
        ++ahead;
        advance(ahead_g, ahead_base);
    };
    for (int i = 0; i < kAhead && i < count; ++i) {
        keep();
        next(i);
    }
    int g = 0;
    for (int n = 0; n < count; ++n) {
        keep();
        held = -1;
        arrived<2 * Copy::kPasses>(kAhead == 2 && ahead == n + 2 && newest_whole);
        const int at = now, before = buffer ? buffer - 1 : kBuffers - 1;
        advance(g, now);
        if (ahead < count) next(before);
        const int qt = buffer * Q::kBytes, gt = (kBuffers + buffer) * Q::kBytes;
        const float *ls = lse[buffer], *de = delta[buffer];
        buffer = buffer + 1 < kBuffers ? buffer + 1 : 0;
        for (int b = 0; b < NB; ++b) {
            const int p0 = at + 32 * b, p1 = p0 + 31;
            if (p0 >= end || p1 < k0 || p0 - k1 >= a.window) continue;
            const bool whole = p1 < end && k1 <= p0 && p1 - k0 < a.window;
            keys.template take<BQ>(
                lds, qt, gt, ls, de, b, at, whole, a.c, [&](int p) { return p < end && p >= key && p - key < a.window; },
                [&](int p) { return p == 0 || (a.window == 1 && a.sinks == 0); });
        }
    }
    // queries behind the window that see the first tokens
    if (first_keys && wave == 0 && key < a.sinks) {
        const float* p = first.part + (int64_t)key * a.dim;
#pragma unroll
        for (int d = 0; d < DP / 32; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int e = 32 * d + acc_row(i, half);
                if (e < a.dim) {
                    keys.dk[d][i] += p[e];
                    keys.dv[d][i] += p[(int64_t)a.sinks * a.dim + e];
                }
            }
    }
    const uint64_t bad_k = __ballot(live && nonfinite(keys.dk)), bad_v = __ballot(live && nonfinite(keys.dv));
    const int64_t to = ((int64_t)(st.first + key) * a.kv_heads + kvh) * a.dim;
#pragma unroll
    for (int b = 0; b < DP / 32; ++b)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const int d = 32 * b + acc_row(i, half);
            if (!live || d >= a.dim) continue;
            put4(static_cast<T*>(a.dk) + to + d, keys.dk[b][i] * a.scale, keys.dk[b][i + 1] * a.scale, keys.dk[b][i + 2] * a.scale, keys.dk[b][i + 3] * a.scale);
            put4(static_cast<T*>(a.dv) + to + d, keys.dv[b][i], keys.dv[b][i + 1], keys.dv[b][i + 2], keys.dv[b][i + 3]);
        }
    if (bad_k | bad_v) {
        const Again b = arguments();
        const int64_t n = die_order(b.block, b.k_items);
        repair_tile<T, DP>(b, seq_tile(b.seq, (int)(n % b.k_places), kGroupCols), (int)(n / b.k_places), threadIdx.x / kWave * kCols,
                       (uint32_t)bad_k | (uint32_t)(bad_k >> 32), (uint32_t)bad_v | (uint32_t)(bad_v >> 32));
    }
}

// ---------------------------------------------------------------------------
// 32 keys a workgroup, each wave 32 queries of a head at a time in its own part
// of LDS, without barriers; the waves' sums are added at the end.  Two uses:
//  - FIRST: the first tokens' keys and the queries that have left them behind
//    their window, a piece of the queries a workgroup; leaves sums for the tile
//    of the sequence's first keys;
//  - otherwise dk and dv of small problems, whose tiles of 128 keys would leave
//    the chip idle: four times the workgroups, and the queries' walk is shared
//    by four waves.
// A block's rows come from memory as it begins: with the next one's in registers
// meanwhile, and operands of one part, 1000 tokens of 16 x 128 took 149 us, not 144, of
// 8 x 256 bf16 315, not 257.
// ---------------------------------------------------------------------------
template <typename T, int DP> constexpr int kNarrowOwn = 2 * Tile<T, DP, 32>::kBytes + 256;      // a wave's queries, gradients, lse and delta
template <typename T, int DP> constexpr int kNarrowWaves = 4 * kNarrowOwn<T, DP> > 160 * 1024 ? 2 : 4;
template <typename T, int DP>
constexpr int kNarrowLds = kNarrowWaves<T, DP> * (kNarrowOwn<T, DP> > 32 * 33 * 4 ? kNarrowOwn<T, DP> : 32 * 33 * 4);

template <typename T, int DP, bool FIRST>
__global__ __launch_bounds__((kNarrowWaves<T, DP> * kWave), (DP * sizeof(T) > 128 ? 1 : 2)) void window_narrow_kernel(AttnBwdArgs a) {
    using Q = Tile<T, DP, 32>;
    constexpr int kRound = 32 * Q::kChunks / kWave, kOwn = kNarrowOwn<T, DP>, NW = kNarrowWaves<T, DP>;
    extern __shared__ __align__(16) char stage[];
    __shared__ uint32_t again[2];      // keys whose dk or dv is not finite
    const int64_t items = (FIRST ? a.pieces : a.k_places) * a.kv_heads, item = die_order(blockIdx.x, items);
    if (item >= items) return;
    const int kvh = (int)(item % a.kv_heads);
    const int place = (int)(item / a.kv_heads);
    const SeqTile st = FIRST ? piece_tile(a, place) : seq_tile(a.seq, place, kCols);
    if (st.row >= st.len) return;
    // the queries' rows
    const int64_t far = FIRST ? (int64_t)st.row + a.piece : (int64_t)st.row + kCols - 1 + a.window;
    const int end = far < st.len ? (int)far : st.len;
    if (FIRST && end <= a.window) return;
    const int from = FIRST && st.row < a.window ? a.window : st.row;
    const int tid = threadIdx.x, wave = uniform(tid / kWave), lane = tid % kWave, half = lane / 32, col = lane % kCols;
    const int group = a.q_heads / a.kv_heads, k0 = FIRST ? 0 : st.row, key = k0 + col;
    const bool live = key < st.len && (!FIRST || key < a.sinks);
    char* own = stage + wave * kOwn;
    float *lse = reinterpret_cast<float*>(own + 2 * Q::kBytes), *delta = lse + 32;
    Keys<T, DP> keys;
    keys.load(static_cast<const T*>(a.k) + (int64_t)(st.first + key) * a.ld_k + (int64_t)kvh * a.dim,
              static_cast<const T*>(a.v) + (int64_t)(st.first + key) * a.ld_v + (int64_t)kvh * a.dim, half, a.dim, live);
    const int blocks = (end - from + 31) / 32;
    const int64_t count = (int64_t)blocks * group;
    Chunk x[kRound], g[kRound];
    float lr = 0.0f, er = 0.0f;
    auto fetch = [&](int64_t n) {
        const int head = kvh * group + (int)(n / blocks), base = from + (int)(n % blocks) * 32;
#pragma unroll
        for (int i = 0; i < kRound; ++i) {
            const int m = lane + i * kWave, p = base + m / Q::kChunks, e = m % Q::kChunks * Q::kElems;
            if (p < end && e < a.dim) {
                x[i].load(static_cast<const T*>(a.q) + (int64_t)(st.first + p) * a.ld_q + (int64_t)head * a.dim + e);
                g[i].load(static_cast<const T*>(a.dy) + ((int64_t)(st.first + p) * a.q_heads + head) * a.dim + e);
            } else {
                x[i].zero();
                g[i].zero();
            }
        }
        const int p = base + col;
        const int64_t at = (int64_t)(st.first + (p < end ? p : end - 1)) * a.q_heads + head;
        lr = a.lse[at] * kLog2e;
        er = a.delta[at];
    };
    for (int64_t n = wave; n < count; n += NW) {
        const int base = from + (int)(n % blocks) * 32;
        fetch(n);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int i = 0; i < kRound; ++i) {
            const int m = lane + i * kWave, to = Q::at(m / Q::kChunks, m % Q::kChunks);
            x[i].store(own + to);
            g[i].store(own + Q::kBytes + to);
        }
        if (lane < 32) lse[lane] = lr, delta[lane] = er;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if constexpr (FIRST) {
            keys.template take<32>(own, 0, Q::kBytes, lse, delta, 0, base, false, a.c,
                                   [&](int p) { return p < end && key < a.sinks && p - key >= a.window; }, [](int) { return false; });
        } else {
            const bool whole = base + 32 <= end && k0 + kCols - 1 <= base && base + 31 - k0 < a.window;
            keys.template take<32>(own, 0, Q::kBytes, lse, delta, 0, base, whole, a.c, [&](int p) { return p < end && p >= key && p - key < a.window; },
                                   [&](int p) { return p == 0 || (a.window == 1 && a.sinks == 0); });
        }
    }
    // the waves' sums, in their order: 32 channels of all keys at a time
    const FirstSums first(a, st, kvh);
    const bool first_keys = !FIRST && st.row == 0 && first.any;
    if (first_keys) first.add(tid, NW * kWave);
    float(*sum)[32][33] = reinterpret_cast<float(*)[32][33]>(stage);      // wave, channel, key
    if (tid < 2) again[tid] = 0;
    __syncthreads();
#pragma unroll
    for (int which = 0; which < 2; ++which)
#pragma unroll
        for (int d = 0; d < DP / 32; ++d) {
#pragma unroll
            for (int i = 0; i < 16; ++i) sum[wave][acc_row(i, half)][col] = which ? keys.dv[d][i] : keys.dk[d][i];
            __syncthreads();
            for (int n = tid; n < 32 * 32; n += NW * kWave) {
                const int e = 32 * d + n % 32, s = n / 32;
                float v = sum[0][n % 32][s];
#pragma unroll
                for (int w = 1; w < NW; ++w) v += sum[w][n % 32][s];
                if (e >= a.dim) continue;
                if constexpr (FIRST) {
                    if (s < a.sinks) a.part[((((int64_t)place * a.kv_heads + kvh) * 2 + which) * a.sinks + s) * a.dim + e] = v;
                } else if (k0 + s < st.len) {
                    if (first_keys && s < a.sinks) v += first.part[(int64_t)(which * a.sinks + s) * a.dim + e];
                    if (!finite(v)) atomicOr(&again[which], 1u << s);
                    const int64_t to = ((int64_t)(st.first + k0 + s) * a.kv_heads + kvh) * a.dim + e;
                    if (which) static_cast<T*>(a.dv)[to] = (T)v;
                    else static_cast<T*>(a.dk)[to] = (T)(v * a.scale);
                }
            }
            __syncthreads();
        }
    if constexpr (!FIRST)
        if (again[0] | again[1]) {
            const Again b = arguments();
            const int64_t n = die_order(b.block, b.k_items);
            const uint32_t mine = (NW == 4 ? 0x11111111u : 0x55555555u) << threadIdx.x / kWave;
            repair_tile<T, DP>(b, seq_tile(b.seq, (int)(n / b.kv_heads), kCols), (int)(n % b.kv_heads), 0, again[0] & mine, again[1] & mine);
        }
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
// Tiles of 128 keys that would leave CUs idle go to the narrow kernel: 2503 tokens
// of 2 heads fp32 (40 tiles) 368 -> 209 us, 1000 tokens of 4 heads bf16 (32) 261 ->
// 176, as they first ran.  Where they fill the chip they are faster: 16384 tokens of 4
// heads bf16 in sequences of 64 (1024 half full) 223 us, 268 in the narrow kernel, of
// 16 331 and 347.  Places are counted, not rows: ragged sequences have up to one each
// more than they fill (4096 tokens in 64 of them 209 us, which the narrow kernel
// would do in 148, 500 in 64 57 and 46).
constexpr int64_t kNarrowBelow = 256;

// Pieces of queries that may see first tokens outside of their window: none
// where no sequence can be longer than the window.
int64_t piece_rows(const im2win_window_desc* d) {
    // some 1024 workgroups, of whole rounds of their waves (512 rows whatever the
    // problem: as they first ran, 1000 tokens 181 us, not 144, 2503 of 2 heads fp32 261, not 188,
    // 16384 of 4 heads 921, not 906)
    const int64_t rows = (d->tokens * d->kv_heads / 1024 + 127) / 128 * 128;
    return std::max<int64_t>(128, std::min<int64_t>(rows, 4096));
}
int64_t pieces_of(const im2win_window_desc* d, const int32_t* starts) {
    if (!d->sinks || d->tokens <= d->window) return 0;
    if (!starts && d->tokens / d->sequences <= d->window) return 0;
    if (!starts) return seq_places(d->tokens, d->sequences, starts, piece_rows(d));
    return d->tokens / piece_rows(d) + std::min(d->sequences, d->tokens / (d->window + 1));
}
// With and without seq_starts (whose places are never fewer): the query does not know.
size_t bwd_bytes(const im2win_window_desc* d) {
    const size_t delta = ((size_t)(d->tokens * d->q_heads) * 4 + 15) / 16 * 16;
    const int64_t pieces = d->sinks && d->tokens > d->window ? d->tokens / piece_rows(d) + std::min(d->sequences, d->tokens / (d->window + 1)) : 0;
    return delta + (size_t)(pieces * d->kv_heads * 2 * d->sinks * d->head_dim) * 4;
}

}  // namespace
}  // namespace im2win

using namespace im2win;

extern "C" {

int im2win_window_attention_backward_workspace_bytes(const im2win_window_desc* d, size_t* bytes) {
    int rc = check_attention(d);
    if (rc) return rc;
    if (d->sequences < 1 || d->sequences > kMaxTokens) return fail(IM2WIN_EINVAL, "sequences must be 1 to %lld (got %lld)", (long long)kMaxTokens, (long long)d->sequences);
    if (!bytes) return fail(IM2WIN_ENULL, "bytes is NULL");
    *bytes = bwd_bytes(d);
    return ok();
}

int im2win_window_attention_backward(const im2win_window_desc* d, const void* dy, const void* q, const void* k, const void* v, const void* y,
                                     const float* lse, const int32_t* seq_starts, void* dq, void* dk, void* dv, void* workspace,
                                     size_t workspace_bytes, void* stream) {
    int rc = check_attention(d);
    if (rc || (rc = check_sequences(d->tokens, d->sequences, seq_starts, true))) return rc;
    if (d->tokens == 0) return ok();
    const size_t e = size_of(d->dtype), need = bwd_bytes(d);
    if ((rc = need_ptr(dy, e, "dy")) || (rc = need_ptr(q, e, "q")) || (rc = need_ptr(k, e, "k")) || (rc = need_ptr(v, e, "v")) ||
        (rc = need_ptr(y, e, "y")) || (rc = need_ptr(lse, 4, "lse")) || (rc = need_ptr(dq, e, "dq")) || (rc = need_ptr(dk, e, "dk")) ||
        (rc = need_ptr(dv, e, "dv")) || (rc = need_ptr(workspace, 16, "workspace")))
        return rc;
    if (workspace_bytes < need) return fail(IM2WIN_EWORKSPACE, "workspace holds %zu bytes, the gradients need %zu", workspace_bytes, need);
    AttnBwdArgs a{};
    a.dy = dy; a.q = q; a.k = k; a.v = v; a.y = y; a.lse = lse; a.dq = dq; a.dk = dk; a.dv = dv;
    a.ld_q = d->ld_q; a.ld_k = d->ld_k; a.ld_v = d->ld_v;
    a.q_heads = (int)d->q_heads; a.kv_heads = (int)d->kv_heads; a.dim = (int)d->head_dim; a.window = (int)d->window; a.sinks = (int)d->sinks;
    a.pack = heads_packed(d->q_heads, d->kv_heads);
    a.tile = kGroupCols / a.pack;
    a.c = d->scale * kLog2e; a.scale = d->scale;
    a.seq = make_seq_map(d->tokens, d->sequences, seq_starts);
    a.q_places = seq_places(d->tokens, d->sequences, seq_starts, a.tile);
    a.q_items = a.q_places * (d->q_heads / a.pack);
    // where tiles of 128 keys would not give every CU a workgroup, tiles of 32
    const bool narrow = seq_places(d->tokens, d->sequences, seq_starts, kGroupCols) * d->kv_heads < kNarrowBelow;
    a.k_places = seq_places(d->tokens, d->sequences, seq_starts, narrow ? kCols : kGroupCols);
    a.k_items = a.k_places * d->kv_heads;
    a.pieces = pieces_of(d, seq_starts);
    a.piece = (int)piece_rows(d);
    a.delta = static_cast<float*>(workspace);
    a.part = reinterpret_cast<float*>(static_cast<char*>(workspace) + ((size_t)(d->tokens * d->q_heads) * 4 + 15) / 16 * 16);
    const int64_t gq = (a.q_items + 7) / 8 * 8, gk = (a.k_items + 7) / 8 * 8, gs = (a.pieces * d->kv_heads + 7) / 8 * 8;
    if ((rc = check_launch(gq, kAttnThreads, "window_attention_backward's queries")) || (rc = check_launch(gk, kAttnThreads, "window_attention_backward's keys")) ||
        (rc = check_launch(gs, kAttnThreads, "window_attention_backward's first tokens")))
        return rc;
    hipStream_t s = static_cast<hipStream_t>(stream);
    hipError_t attribute = hipSuccess;
    with_type(d->dtype, [&](auto ty) {
        using T = decltype(ty);
        with_head(d->head_dim, [&](auto dp) {
            constexpr int DP = decltype(dp)::value;
            constexpr int kLds = kNarrowLds<T, DP>;
            auto allow = [&](const void* kernel) {
                if (kLds > 65536 && attribute == hipSuccess) attribute = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
            };
            if (a.pieces) allow(reinterpret_cast<const void*>(&window_narrow_kernel<T, DP, true>));
            if (narrow) allow(reinterpret_cast<const void*>(&window_narrow_kernel<T, DP, false>));
            if (attribute != hipSuccess) return;
            hipLaunchKernelGGL((window_dq_kernel<T, DP>), dim3((unsigned)gq), dim3(kAttnThreads), 0, s, a);
            constexpr int kThreads = kNarrowWaves<T, DP> * kWave;
            if (a.pieces) hipLaunchKernelGGL((window_narrow_kernel<T, DP, true>), dim3((unsigned)gs), dim3(kThreads), kLds, s, a);
            if (narrow) hipLaunchKernelGGL((window_narrow_kernel<T, DP, false>), dim3((unsigned)gk), dim3(kThreads), kLds, s, a);
            else hipLaunchKernelGGL((window_dkv_kernel<T, DP>), dim3((unsigned)gk), dim3(kAttnThreads), 0, s, a);
        });
    });
    if (attribute != hipSuccess) return fail(IM2WIN_EHIP, "window_attention_backward's LDS: %s", hipGetErrorString(attribute));
    return launched("window_attention_backward");
}

}  // extern "C"
