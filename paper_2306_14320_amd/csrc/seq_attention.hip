// Attention with a sliding window and a few first tokens that stay visible,
// over packed sequences, and its form for single tokens.  For a query at
// position p of its sequence,
//   y = sum_j w_j v_j,  w = softmax_j(scale q k_j),
// over the keys j <= p with j > p - window or j < sinks.
//
// One pass over the visible keys with the running maximum m and sum l of the
// softmax; scores and weights never leave the registers.  Keys of positions
// the request had before the call come from its cache, a ring of sinks +
// window rows, in which the call leaves the new tokens' keys and values.
//
// 16384 tokens of 16 heads over 4, 128 bf16 channels, window 1024, in front of the
// gradients: 227 us, where three products (the weights have two parts) would take
// 161 at the rate of a large one; matrix cores are busy for 44%, vector units for
// 51%, and waves wait for 36% of their cycles.  9001 tokens of 12 heads over 4, 64
// channels, window 500, 13 ragged prompts: 47 us (17 for the products), and 5 for
// the caches; vector units 61%, matrix cores 25%: exponentials, maximum, sum and
// both parts of 64 channels' weights take longer than their products.
#include "seq_attention.h"

#include <algorithm>

namespace im2win {
namespace {

struct AttnArgs {
    const void *q, *k, *v;
    void *k_cache, *v_cache;
    const int32_t *past, *slots;
    void* y;
    float* lse;
    SeqMap seq;
    int64_t ld_q, ld_k, ld_v, cache_slots;
    int64_t places, items;
    int q_heads, kv_heads, dim, window, sinks;
    int pack, tile;          // heads of a workgroup, its queries
    float c;                 // scale log2(e)
    // single tokens
    int requests, splits, split_rows, stage;
    float *part_ml, *part_o;
};

constexpr int kMaxPast = 1 << 30;

__device__ __forceinline__ int past_of(const int32_t* past, int b) {
    const int p = past ? uniform(past[b]) : 0;
    return p < 0 ? 0 : p > kMaxPast ? kMaxPast : p;
}
// The row of position p in a request's cache
__device__ __forceinline__ int ring(int p, int window, int sinks) { return p < sinks ? p : sinks + (p - sinks) % window; }

// Running softmax of a lane's column and its output
template <int DP>
struct Running {
    float m = -INFINITY, l = 0.0f;
    f32x16 o[DP / 32];
    __device__ __forceinline__ Running() {
#pragma unroll
        for (int t = 0; t < DP / 32; ++t) o[t] = f32x16{};
    }
};

// Takes NB blocks of 32 masked scores (raw products) into the running softmax
// and leaves the weights in their place.  The base of the exponentials, m, need
// not be the largest score: it is moved where a score passes it by more than
// 2^8, so that most tiles leave the sums as they are.
template <int DP, int NB>
__device__ __forceinline__ void soften(Running<DP>& r, f32x16 (&s)[NB], float c) {
    float top = s[0][0];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, s[b][i]);
    top = half_max(top) * c;
    if (__ballot(top > r.m + 8.0f)) {
        const float m = top > r.m + 8.0f ? top : r.m;
        const float a = __builtin_amdgcn_exp2f(r.m - (m == -INFINITY ? 0.0f : m));      // 0 in a column that has seen no key yet
        r.m = m;
        r.l *= a;
#pragma unroll
        for (int t = 0; t < DP / 32; ++t) r.o[t] *= a;
    }
    const float base = r.m == -INFINITY ? 0.0f : r.m;
    float sum = 0.0f;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            s[b][i] = __builtin_amdgcn_exp2f(fmaf(s[b][i], c, -base));
            sum += s[b][i];
        }
    r.l += sum;       // of the lane's half; the halves are added at the end
}

// Keys of a tile.  9001 tokens of 12 heads of 64 channels take 51.7 us with 64 keys,
// 53.5 with 32, but 16384 of 16 heads of 128 channels 420 and 242: two buffers of 64
// such rows leave LDS for two workgroups.  (32 rows of 32 or 96 channels are no whole
// number of copies by all threads.)
template <typename T, int DP> constexpr int kTileKeys = sizeof(T) == 2 && DP <= 96 ? 64 : 32;
// Waves a SIMD.  Of 128 channels of bf16 three hide the waits for LDS best (16384 tokens
// of 16 heads, window 1024: 242 us, 254 with two), of 64 and fewer four (9001 tokens of
// 12 heads: 52 us, 58 with three); of 96 three gain nothing over two, and wider rows
// have registers for two, or one.
template <typename T, int DP> constexpr int kFwdWaves = DP * sizeof(T) > 384 || DP >= 192 ? 1 : sizeof(T) == 2 && DP != 96 ? (DP > 64 ? 3 : 4) : 2;
// The step: waves a SIMD, and whether the next rows wait in registers while
// some are worked on (beside 1 KB of queries and outputs a lane they would spill).
constexpr int step_waves(int row_bytes) { return row_bytes <= 128 ? 4 : row_bytes <= 256 ? 2 : 1; }
template <typename T, int DP> constexpr bool kStepAhead = DP * sizeof(T) <= 512 && DP <= 192;
// A wave's LDS for 32 rows: keys and values, or values in the place of keys
template <typename T, int DP> constexpr int kStepStage = (kStepAhead<T, DP> ? 2 : 1) * Tile<T, DP, 32>::kBytes;

// ---------------------------------------------------------------------------
// Prompts and training: a workgroup takes up to 128 columns, the queries of
// `tile` rows for `pack` heads that share keys and values.  Their tiles pass
// through LDS, the next one's copies under way while one is worked on.
// ---------------------------------------------------------------------------
template <typename T, int DP>
__global__ __launch_bounds__(kAttnThreads, (kFwdWaves<T, DP>)) void window_attention_kernel(AttnArgs a) {
    constexpr int BK = kTileKeys<T, DP>, NB = BK / 32;
    using KV = Tile<T, DP, BK>;
    using Copy = Feed<T, DP, BK>;
    constexpr int kAhead = kAheadTiles<KV::kBytes, kFwdWaves<T, DP>>, kBuffers = kAhead + 1;
    __shared__ __align__(128) char lds[2 * kBuffers * KV::kBytes];      // buffers of keys, then of values
    __shared__ uint32_t flags[kBuffers][2];      // rows of a buffer whose values are not all finite
    const int64_t item = die_order(blockIdx.x, a.items);
    if (item >= a.items) return;
    const int hb = (int)(item / a.places);
    const SeqTile st = seq_tile(a.seq, (int)(item % a.places), a.tile);
    if (st.row >= st.len) return;
    const int tid = threadIdx.x, wave = uniform(tid / kWave), lane = tid % kWave, half = lane / 32;
    const int h0 = hb * a.pack, kvh = h0 / (a.q_heads / a.kv_heads);
    const int rows = a.sinks + a.window;
    const int64_t slot = !a.k_cache ? 0 : a.slots ? uniform(a.slots[st.b]) : st.b;
    const bool served = !a.k_cache || (slot >= 0 && slot < a.cache_slots);
    const int past = a.k_cache ? past_of(a.past, st.b) : 0;

    // the lane's column
    const int col = wave * kCols + lane % kCols, qi = col / a.pack;
    const int row = st.row + qi;                        // of the sequence
    const bool live = qi < a.tile && row < st.len;
    const int last = st.row + a.tile < st.len ? st.row + a.tile - 1 : st.len - 1;
    const int pos = past + (row < last ? row : last);
    const int head = h0 + col % a.pack;
    Frag<T> q[DP / 16];
    {
        const T* p = static_cast<const T*>(a.q) + (st.first + (row < last ? row : last)) * a.ld_q + (int64_t)head * a.dim;
#pragma unroll
        for (int s = 0; s < DP / 16; ++s) {
            if (16 * s + 8 * half < a.dim) q[s].load(p + 16 * s + 8 * half);
            else q[s].zero();
        }
    }

    // the keys: where sinks lie in front of the first query's window a tile of them, then the window's
    const int qfirst = past + st.row, qlast = past + last;
    const int begin = qfirst - a.window + 1 > 0 ? qfirst - a.window + 1 : 0;
    const int first_end = a.sinks < begin ? a.sinks : begin;      // keys of the sinks' tile
    const int end = qlast + 1;
    // queries of this wave, for tiles that all of them see
    const int wq0 = past + st.row + wave * kCols / a.pack;
    int wq1 = past + st.row + (wave * kCols + kCols - 1) / a.pack;
    wq1 = wq1 < qlast ? wq1 : qlast;

    // the value or key rows of the call, from position `past` on, and those of the cache
    auto cached = [&](int p) { return ((slot * rows + ring(p, a.window, a.sinks)) * a.kv_heads + kvh) * a.dim; };
    const Copy ck(a.ld_k), cv(a.ld_v);
    const char* kn = reinterpret_cast<const char*>(static_cast<const T*>(a.k) + st.first * a.ld_k + (int64_t)kvh * a.dim);
    const char* vn = reinterpret_cast<const char*>(static_cast<const T*>(a.v) + st.first * a.ld_v + (int64_t)kvh * a.dim);
    auto value = [&](int p) {
        return p < past ? static_cast<const T*>(a.v_cache) + cached(p) : reinterpret_cast<const T*>(vn + (int64_t)(p - past) * cv.stride);
    };
    auto issue = [&](int buffer, int base, int stop) {
        char *kt = lds + buffer * KV::kBytes, *vt = lds + (kBuffers + buffer) * KV::kBytes;
        if (base >= past) {
            ck.issue(kt, kn + (int64_t)(base - past) * ck.stride, stop - base, a.dim);
            cv.issue(vt, vn + (int64_t)(base - past) * cv.stride, stop - base, a.dim);
            return;
        }
#pragma unroll
        for (int i = 0; i < Copy::kPasses; ++i) {
            const int n = base + Copy::row(i), p = n < stop ? n : stop - 1, e = Copy::chunk(i) * KV::kElems;
            if (e >= a.dim) continue;
            const T* k = p < past ? static_cast<const T*>(a.k_cache) + cached(p) : reinterpret_cast<const T*>(kn + (int64_t)(p - past) * ck.stride);
            Copy::copy(k + e, kt, i);
            Copy::copy(value(p) + e, vt, i);
        }
    };

    const int rb = KV::row_base(lane), cb = KV::col_base(lane);
    Running<DP> r;
    if (a.dim != DP) clear(lds, 2 * kBuffers * KV::kBytes);
    if (tid < 2 * kBuffers) flags[tid / 2][tid % 2] = 0;
    // tile i: the sinks', where there is one, and those of the windows
    const int lead = first_end > 0 ? 1 : 0, count = served ? lead + (end - begin + BK - 1) / BK : 0;
    auto base_of = [&](int i) { return i < lead ? 0 : begin + (i - lead) * BK; };
    auto stop_of = [&](int i) { return i < lead ? first_end : end; };
    for (int i = 0; i < kAhead && i < count; ++i) issue(i, base_of(i), stop_of(i));
    int buffer = 0;
    for (int n = 0; n < count; ++n) {
        const bool sink_tile = n < lead;
        const int now = base_of(n), now_stop = stop_of(n), newest = n + kAhead - 1;
        // the newest tile under way, if it is another: whole, and not of the cache, it is as many copies in every wave
        arrived<2 * Copy::kPasses>(kAhead == 2 && newest < count && a.dim == DP && base_of(newest) >= past && base_of(newest) + BK <= stop_of(newest));
        // a tile that some column does not see all of: its values' infinities and NaN stay out of the product
        if (now + BK > now_stop || now + BK - 1 > qfirst || now <= qlast - a.window) {
            bool bad = false;
#pragma unroll
            for (int i = 0; i < Copy::kPasses; ++i) {
                Chunk c;
                c.load(lds + (kBuffers + buffer) * KV::kBytes + (tid + i * kAttnThreads) * 16);
                bad |= nonfinite<T>(c);
            }
            if (bad) {
#pragma unroll
                for (int i = 0; i < Copy::kPasses; ++i) {
                    char* to = lds + (kBuffers + buffer) * KV::kBytes + (tid + i * kAttnThreads) * 16;
                    Chunk c;
                    c.load(to);
                    if (!nonfinite<T>(c)) continue;
                    drop_nonfinite<T>(c);
                    c.store(to);
                    atomicOr(&flags[buffer][Copy::row(i) / 32], 1u << Copy::row(i) % 32);
                }
            }
            __syncthreads();
        }
        const int current = buffer, before = buffer ? buffer - 1 : kBuffers - 1;      // the tile before was read in front of the last barrier
        if (tid < 2) flags[before][tid] = 0;
        if (n + kAhead < count) issue(before, base_of(n + kAhead), stop_of(n + kAhead));
        const int kb = rb + buffer * KV::kBytes, vb = cb + (kBuffers + buffer) * KV::kBytes;
        buffer = buffer + 1 < kBuffers ? buffer + 1 : 0;
#pragma unroll
        for (int b = 0; b < NB; ++b) {      // 32 keys at a time
            // those in front of the wave's first window (but for sinks) or behind its last query
            const int from = now + 32 * b;
            if (from > wq1 || (from + 32 <= wq0 - a.window + 1 && from >= a.sinks) || (b && sink_tile)) continue;
            f32x16 s[1] = {f32x16{}};
#pragma unroll
            for (int d = 0; d < DP / 16; ++d) mma(s[0], KV::row_frag(lds, kb, b, d), q[d]);
            if (sink_tile) {                // all of them seen, by all
                const int n = now_stop - 4 * half;
#pragma unroll
                for (int i = 0; i < 16; ++i) s[0][i] = 32 * b + acc_row(i, 0) < n ? s[0][i] : -INFINITY;
            } else if (now < a.sinks) {     // the sequence's first keys
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int p = now + 32 * b + acc_row(i, half);
                    s[0][i] = p <= pos && (p > pos - a.window || p < a.sinks) ? s[0][i] : -INFINITY;
                }
            } else if (!(from + 31 <= wq0 && from > wq1 - a.window)) {      // pos - window < p <= pos
                const int low = pos - a.window + 1 - now - 4 * half;
#pragma unroll
                for (int i = 0; i < 16; ++i) s[0][i] = (uint32_t)(32 * b + acc_row(i, 0) - low) < (uint32_t)a.window ? s[0][i] : -INFINITY;
            }
            soften<DP, 1>(r, s, a.c);
            __builtin_amdgcn_s_setprio(1);      // a wave with products to issue goes first
#pragma unroll
            for (int part = 0; part < 2; ++part) {
                const Weights<T> w(s[0], part);
#pragma unroll
                for (int t = 0; t < DP / 32; ++t) mma(r.o[t], KV::col_frag(lds, vb, t, 2 * b + part), w);
            }
            __builtin_amdgcn_s_setprio(0);
        }
        // what was kept out of the product: a column that sees such a value has it
        for (int f = 0; f < NB; ++f)
            for (uint32_t rest = uniform(flags[current][f]); rest; rest &= rest - 1) {
                const int p = now + 32 * f + __builtin_ctz(rest);
                if (p >= now_stop) continue;      // the last row again
                const bool seen = p <= pos && (p > pos - a.window || p < a.sinks);
                const T* v = value(p);
                uint32_t dim = a.dim;      // not known to be the kernel's: comparisons of every channel would be kept from the start
                arrive(dim);
#pragma unroll
                for (int t = 0; t < DP / 32; ++t)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const uint32_t d = 32 * t + acc_row(i, half);
                        if (d < dim && seen && !finite(v[d])) r.o[t][i] += (float)v[d];
                    }
            }
    }
    const float l = half_sum(r.l);
    if (!live) return;
    // A query sees itself, so a served one's l is zero only where all of its scores are
    // -inf: 0 / 0 then, as the softmax has it.
    const float scale = served ? 1.0f / l : 0.0f;
    const int64_t t = st.first + row;
    T* y = static_cast<T*>(a.y) + (t * a.q_heads + head) * a.dim;
#pragma unroll
    for (int b = 0; b < DP / 32; ++b)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const int d = 32 * b + acc_row(i, half);
            if (d < a.dim) put4(y + d, r.o[b][i] * scale, r.o[b][i + 1] * scale, r.o[b][i + 2] * scale, r.o[b][i + 3] * scale);
        }
    if (a.lse && half == 0) a.lse[t * a.q_heads + head] = l == 0.0f ? -INFINITY : (r.m + __builtin_amdgcn_logf(l)) * kLn2;
}

// The cache behind a prompt: a wave takes a new token, and copies its keys and
// values where they are among the first tokens or the last window.
template <typename T>
__global__ __launch_bounds__(kAttnThreads) void window_cache_kernel(AttnArgs a) {
    const int t = uniform((int)(blockIdx.x * 4 + threadIdx.x / kWave)), lane = threadIdx.x % kWave;
    if (t < a.seq.first(0) || t >= a.seq.first(a.seq.count)) return;
    const SeqMap::Found f = a.seq.at(t);
    const int64_t slot = a.slots ? uniform(a.slots[f.b]) : f.b;
    if (slot < 0 || slot >= a.cache_slots) return;
    const int past = past_of(a.past, f.b), p = past + t - f.first, end = past + f.end - f.first;
    if (p >= a.sinks && p < end - a.window) return;
    const int n = a.kv_heads * a.dim;
    const int64_t to = (slot * (a.sinks + a.window) + ring(p, a.window, a.sinks)) * n;
    constexpr int E = 16 / sizeof(T);
    for (int e = lane * E; e < n; e += kWave * E) {
        Chunk k, v;
        k.load(static_cast<const T*>(a.k) + t * a.ld_k + e);
        v.load(static_cast<const T*>(a.v) + t * a.ld_v + e);
        k.store(static_cast<T*>(a.k_cache) + to + e);
        v.store(static_cast<T*>(a.v_cache) + to + e);
    }
}

// ---------------------------------------------------------------------------
// Single tokens: the columns are the heads of a request that share keys and
// values; a workgroup takes a share of its cache's rows, each wave 32 of them at
// a time, whole rows by neighbouring lanes, through its own part of LDS.  The
// new token's row is read from the inputs and written to the cache by the lanes
// that hold it.  Bound by memory: 128 requests of 1028 rows of 4 heads of 128 bf16
// take 49 us, 4.5 TB/s (with each lane reading its own row 56, when it took 47 to
// 48.6 with weights of one part).  In fp32 the matrix instructions bound it, of
// which a request's 4 heads use 4 columns of 32: 141 us, 87 at a copy's rate.
// ---------------------------------------------------------------------------
template <typename T, int DP>
__global__ __launch_bounds__(kAttnThreads, (step_waves(DP * sizeof(T)))) void window_step_kernel(AttnArgs a) {
    using V = Tile<T, DP, 32>;
    constexpr int kRound = 32 * V::kChunks / kWave, NW = kAttnThreads / kWave;      // chunks of a lane; waves
    extern __shared__ __align__(16) char stage[];        // a.stage bytes of each wave
    __shared__ float ml[NW][2][kCols];
    const int tid = threadIdx.x, wave = uniform(tid / kWave), lane = tid % kWave, half = lane / 32;
    const int blocks = a.q_heads / a.pack;
    const int split = blockIdx.x % a.splits, hb = blockIdx.x / a.splits % blocks, b = blockIdx.x / a.splits / blocks;
    const int h0 = hb * a.pack, kvh = h0 / (a.q_heads / a.kv_heads);
    const int64_t rows = a.sinks + a.window, slot = a.slots ? uniform(a.slots[b]) : b;
    const bool served = slot >= 0 && slot < a.cache_slots;
    const int past = past_of(a.past, b), fresh = ring(past, a.window, a.sinks);
    const int filled = !served ? 0 : past + 1 < rows ? past + 1 : (int)rows;
    const int from = split * a.split_rows, to = from + a.split_rows < filled ? from + a.split_rows : filled;
    const int col = lane % kCols, head = h0 + (col < a.pack ? col : 0);
    const int64_t cached = (slot * rows * a.kv_heads + kvh) * a.dim, step = (int64_t)a.kv_heads * a.dim;
    T* kc = static_cast<T*>(a.k_cache) + (served ? cached : 0);
    T* vc = static_cast<T*>(a.v_cache) + (served ? cached : 0);
    const T* kn = static_cast<const T*>(a.k) + b * a.ld_k + (int64_t)kvh * a.dim;
    const T* vn = static_cast<const T*>(a.v) + b * a.ld_v + (int64_t)kvh * a.dim;
    char* mine = stage + wave * a.stage;
    const int cb = V::col_base(lane);

    Frag<T> q[DP / 16];
    const T* qp = static_cast<const T*>(a.q) + b * a.ld_q + (int64_t)head * a.dim;
#pragma unroll
    for (int s = 0; s < DP / 16; ++s) {
        if (16 * s + 8 * half < a.dim) q[s].load(qp + 16 * s + 8 * half);
        else q[s].zero();
    }
    Chunk k[kRound], v[kRound];
    auto fetch = [&](Chunk (&c)[kRound], int base, const T* cache, const T* now) {
#pragma unroll
        for (int i = 0; i < kRound; ++i) {
            const int n = lane + i * kWave, rw = base + n / V::kChunks, e = n % V::kChunks * V::kElems;
            if (rw < to && e < a.dim) c[i].load((rw == fresh ? now : cache + rw * step) + e);
            else c[i].zero();
        }
    };
    // to the wave's LDS; the new token's row to the cache too
    auto put = [&](const Chunk (&c)[kRound], int base, char* lds, T* cache) {
        const bool has_fresh = fresh >= base && fresh < base + 32;
#pragma unroll
        for (int i = 0; i < kRound; ++i) {
            const int n = lane + i * kWave, rw = n / V::kChunks, e = n % V::kChunks * V::kElems;
            if (has_fresh && base + rw == fresh && e < a.dim) c[i].store(cache + fresh * step + e);
            c[i].store(lds + V::at(rw, n % V::kChunks));
        }
    };
    constexpr bool kAhead = kStepAhead<T, DP>;
    const int rb = V::row_base(lane);
    char* values = mine + kStepStage<T, DP> - V::kBytes;
    Running<DP> r;
    const int first = from + wave * 32;
    if (kAhead && first < to) {
        fetch(k, first, kc, kn);
        fetch(v, first, vc, vn);
    }
    for (int base = first; base < to; base += 32 * NW) {
        if (!kAhead) fetch(k, base, kc, kn);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        put(k, base, mine, kc);
        if (kAhead) put(v, base, values, vc);
        else fetch(v, base, vc, vn);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (kAhead && base + 32 * NW < to) {
            fetch(k, base + 32 * NW, kc, kn);
            fetch(v, base + 32 * NW, vc, vn);
        }
        f32x16 s[1] = {f32x16{}};
#pragma unroll
        for (int d = 0; d < DP / 16; ++d) mma(s[0], V::row_frag(mine, rb, 0, d), q[d]);
        if (!kAhead) {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            put(v, base, values, vc);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
        if (base + 32 > to) {
#pragma unroll
            for (int i = 0; i < 16; ++i) s[0][i] = base + acc_row(i, half) < to ? s[0][i] : -INFINITY;
        }
        soften<DP, 1>(r, s, a.c);
#pragma unroll
        for (int part = 0; part < 2; ++part) {
            const Weights<T> w(s[0], part);
#pragma unroll
            for (int t = 0; t < DP / 32; ++t) mma(r.o[t], V::col_frag(values, cb, t, part), w);
        }
    }
    // the four waves' shares: a channel's row of columns each, and their statistics
    r.l = half_sum(r.l);
    float* o = reinterpret_cast<float*>(mine);
#pragma unroll
    for (int t = 0; t < DP / 32; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (col < a.pack) o[(32 * t + acc_row(i, half)) * a.pack + col] = r.o[t][i];
    if (half == 0) ml[wave][0][col] = r.m, ml[wave][1][col] = r.l;
    __syncthreads();
    for (int n = tid; n < a.dim * a.pack; n += kAttnThreads) {
        const int c = n % a.pack, d = n / a.pack;
        float m = -INFINITY;
#pragma unroll
        for (int w = 0; w < NW; ++w) m = fmaxf(m, ml[w][0][c]);
        const float base = m == -INFINITY ? 0.0f : m;
        float sum = 0.0f, l = 0.0f;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float f = __builtin_amdgcn_exp2f(ml[w][0][c] - base);
            l = fmaf(ml[w][1][c], f, l);
            sum = fmaf(reinterpret_cast<const float*>(stage + w * a.stage)[d * a.pack + c], f, sum);
        }
        const int64_t at = (int64_t)b * a.q_heads + h0 + c;
        if (a.splits == 1) {
            static_cast<T*>(a.y)[at * a.dim + d] = (T)(served ? sum / l : 0.0f);
        } else {
            a.part_o[(at * a.splits + split) * a.dim + d] = sum;
            if (d == 0) a.part_ml[(at * a.splits + split) * 2] = m, a.part_ml[(at * a.splits + split) * 2 + 1] = l;
        }
    }
}

// The shares of a request's head: a wave, four channels a lane
template <typename T>
__global__ __launch_bounds__(kAttnThreads) void window_step_join_kernel(AttnArgs a) {
    const int64_t at = (int64_t)blockIdx.x * 4 + threadIdx.x / kWave;
    const int lane = threadIdx.x % kWave;
    if (at >= (int64_t)a.requests * a.q_heads) return;
    const float* ml = a.part_ml + at * a.splits * 2;
    const float* part = a.part_o + at * a.splits * a.dim;
    // the largest of all shares, a share a lane
    float m = -INFINITY;
    for (int s = lane; s < a.splits; s += kWave) m = fmaxf(m, ml[2 * s]);
#pragma unroll
    for (int x = 1; x < kWave; x *= 2) m = fmaxf(m, __shfl_xor(m, x));
    const float base = m == -INFINITY ? 0.0f : m;
    float l = 0.0f, o[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    const int d = 4 * lane < a.dim ? 4 * lane : 0;
    for (int s0 = 0; s0 < a.splits; s0 += kWave) {
        const int n = a.splits - s0 < kWave ? a.splits - s0 : kWave;
        const float f = lane < n ? __builtin_amdgcn_exp2f(ml[2 * (s0 + lane)] - base) : 0.0f;
        l += lane < n ? f * ml[2 * (s0 + lane) + 1] : 0.0f;
#pragma unroll 8
        for (int s = 0; s < n; ++s) {
            const float fs = __shfl(f, s);
            float v[4];
            __builtin_memcpy(v, part + (int64_t)(s0 + s) * a.dim + d, 16);
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = fmaf(v[i], fs, o[i]);
        }
    }
#pragma unroll
    for (int x = 1; x < kWave; x *= 2) l += __shfl_xor(l, x);
    const int b = uniform((int)(at / a.q_heads));
    const int64_t slot = a.slots ? uniform(a.slots[b]) : b;
    const float scale = slot >= 0 && slot < a.cache_slots ? 1.0f / l : 0.0f;
    if (4 * lane < a.dim) put4(static_cast<T*>(a.y) + at * a.dim + d, o[0] * scale, o[1] * scale, o[2] * scale, o[3] * scale);
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
AttnArgs args_of(const im2win_window_desc* d, const void* q, const void* k, const void* v) {
    AttnArgs a{};
    a.q = q; a.k = k; a.v = v;
    a.ld_q = d->ld_q; a.ld_k = d->ld_k; a.ld_v = d->ld_v;
    a.q_heads = (int)d->q_heads; a.kv_heads = (int)d->kv_heads; a.dim = (int)d->head_dim;
    a.window = (int)d->window; a.sinks = (int)d->sinks;
    a.c = d->scale * kLog2e;
    a.pack = heads_packed(d->q_heads, d->kv_heads);
    a.tile = kGroupCols / a.pack;
    return a;
}

int check_cache(const im2win_window_desc* d, const void* k_cache, const void* v_cache, int64_t cache_slots, const int32_t* past, const int32_t* slots) {
    const size_t e = size_of(d->dtype);
    int rc;
    if (cache_slots < 0) return fail(IM2WIN_EINVAL, "cache_slots must be >= 0 (got %lld)", (long long)cache_slots);
    if ((rc = need_ptr(k_cache, e, "k_cache")) || (rc = need_ptr(v_cache, e, "v_cache")) || (rc = may_ptr(slots, 4, "slots"))) return rc;
    return may_ptr(past, 4, "past");
}

// Shares of a request's rows: as many as have room on the chip at once beside the
// other requests' and heads', of 128 rows (one round of the workgroup) at least:
// 100 requests of 260 rows take 16 us, 27 with one share more, which waits for the
// others.  2 requests of 4100 rows have 33 shares: 7.6 us, and 10 for the join.
struct Split {
    int splits, rows;
};
Split split_of(const im2win_window_desc* d) {
    const int64_t blocks = d->tokens * (d->q_heads / heads_packed(d->q_heads, d->kv_heads)), rows = d->sinks + d->window;
    int64_t room = 256;
    with_head(d->head_dim, [&](auto dp) { room = 256 * step_waves((int)(decltype(dp)::value * size_of(d->dtype))); });
    const int64_t n = std::max<int64_t>(1, std::min(blocks ? room / blocks : 1, (rows + 127) / 128));
    Split s{};
    s.rows = (int)(((rows + n - 1) / n + 31) / 32 * 32);
    s.splits = (int)((rows + s.rows - 1) / s.rows);
    return s;
}
size_t step_bytes(const im2win_window_desc* d) {
    const Split s = split_of(d);
    if (s.splits == 1) return 0;
    return (size_t)(d->tokens * d->q_heads * s.splits) * (size_t)(d->head_dim + 2) * 4;
}

}  // namespace
}  // namespace im2win

using namespace im2win;

extern "C" {

int im2win_window_attention(const im2win_window_desc* d, const void* q, const void* k, const void* v, const int32_t* seq_starts,
                            void* k_cache, void* v_cache, int64_t cache_slots, const int32_t* past, const int32_t* slots, void* y, float* lse,
                            void* stream) {
    int rc = check_attention(d);
    if (rc || (rc = check_sequences(d->tokens, d->sequences, seq_starts, true))) return rc;
    const bool cached = k_cache || v_cache;
    if (cached && (rc = check_cache(d, k_cache, v_cache, cache_slots, past, slots))) return rc;
    if (!cached && (past || slots)) return fail(IM2WIN_EINVAL, "past and slots belong to a cache (k_cache is NULL)");
    if (d->tokens == 0) return ok();
    const size_t e = size_of(d->dtype);
    if ((rc = need_ptr(q, e, "q")) || (rc = need_ptr(k, e, "k")) || (rc = need_ptr(v, e, "v")) || (rc = need_ptr(y, e, "y")) || (rc = may_ptr(lse, 4, "lse"))) return rc;
    AttnArgs a = args_of(d, q, k, v);
    a.k_cache = k_cache; a.v_cache = v_cache; a.cache_slots = cache_slots; a.past = past; a.slots = slots;
    a.y = y; a.lse = lse;
    a.seq = make_seq_map(d->tokens, d->sequences, seq_starts);
    a.places = seq_places(d->tokens, d->sequences, seq_starts, a.tile);
    a.items = a.places * (d->q_heads / a.pack);
    const int64_t groups = (a.items + 7) / 8 * 8, copies = (d->tokens + 3) / 4;
    if ((rc = check_launch(groups, kAttnThreads, "window_attention")) || (rc = check_launch(copies, kAttnThreads, "window_attention's cache"))) return rc;
    hipStream_t s = static_cast<hipStream_t>(stream);
    with_type(d->dtype, [&](auto t) {
        using T = decltype(t);
        with_head(d->head_dim, [&](auto dp) {
            hipLaunchKernelGGL((window_attention_kernel<T, decltype(dp)::value>), dim3((unsigned)groups), dim3(kAttnThreads), 0, s, a);
        });
        if (cached) hipLaunchKernelGGL((window_cache_kernel<T>), dim3((unsigned)copies), dim3(kAttnThreads), 0, s, a);
    });
    return launched("window_attention");
}

int im2win_window_attention_step_workspace_bytes(const im2win_window_desc* d, size_t* bytes) {
    int rc = check_attention(d);
    if (rc) return rc;
    if (!bytes) return fail(IM2WIN_ENULL, "bytes is NULL");
    *bytes = step_bytes(d);
    return ok();
}

int im2win_window_attention_step(const im2win_window_desc* d, const void* q, const void* k, const void* v, void* k_cache, void* v_cache,
                                 int64_t cache_slots, const int32_t* past, const int32_t* slots, void* y, void* workspace, size_t workspace_bytes,
                                 void* stream) {
    int rc = check_attention(d);
    if (rc) return rc;
    if (d->tokens == 0) return ok();
    const size_t e = size_of(d->dtype), need = step_bytes(d);
    if ((rc = need_ptr(q, e, "q")) || (rc = need_ptr(k, e, "k")) || (rc = need_ptr(v, e, "v")) || (rc = need_ptr(y, e, "y")) ||
        (rc = check_cache(d, k_cache, v_cache, cache_slots, past, slots)) || (rc = need_ptr(past, 4, "past")) ||
        (need && (rc = need_ptr(workspace, 16, "workspace"))))
        return rc;
    if (workspace_bytes < need) return fail(IM2WIN_EWORKSPACE, "workspace holds %zu bytes, the step needs %zu", workspace_bytes, need);
    AttnArgs a = args_of(d, q, k, v);
    a.k_cache = k_cache; a.v_cache = v_cache; a.cache_slots = cache_slots; a.past = past; a.slots = slots;
    a.y = y;
    const Split sp = split_of(d);
    a.requests = (int)d->tokens; a.splits = sp.splits; a.split_rows = sp.rows;
    a.part_o = static_cast<float*>(workspace);
    a.part_ml = a.part_o + d->tokens * d->q_heads * sp.splits * d->head_dim;
    const int64_t groups = d->tokens * (d->q_heads / a.pack) * sp.splits, joins = (d->tokens * d->q_heads + 3) / 4;
    if ((rc = check_launch(groups, kAttnThreads, "window_attention_step")) || (rc = check_launch(joins, kAttnThreads, "window_attention_step's shares"))) return rc;
    hipStream_t s = static_cast<hipStream_t>(stream);
    hipError_t attribute = hipSuccess;
    with_type(d->dtype, [&](auto t) {
        using T = decltype(t);
        with_head(d->head_dim, [&](auto dp) {
            constexpr int DP = decltype(dp)::value;
            // a wave's keys and values of 32 rows, and behind them its share of the outputs
            a.stage = std::max(kStepStage<T, DP>, a.pack * DP * 4);
            if (4 * a.stage > 65536)
                attribute = hipFuncSetAttribute(reinterpret_cast<const void*>(&window_step_kernel<T, DP>), hipFuncAttributeMaxDynamicSharedMemorySize, 4 * a.stage);
            if (attribute == hipSuccess)
                hipLaunchKernelGGL((window_step_kernel<T, DP>), dim3((unsigned)groups), dim3(kAttnThreads), 4 * a.stage, s, a);
        });
        if (sp.splits > 1 && attribute == hipSuccess)
            hipLaunchKernelGGL((window_step_join_kernel<T>), dim3((unsigned)joins), dim3(kAttnThreads), 0, s, a);
    });
    if (attribute != hipSuccess) return fail(IM2WIN_EHIP, "window_attention_step's LDS: %s", hipGetErrorString(attribute));
    return launched("window_attention_step");
}

}  // extern "C"
