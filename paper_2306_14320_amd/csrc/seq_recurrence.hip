// Gated linear recurrence over packed rows of tokens, its gradients and its
// form for single tokens.  For each channel, along each sequence, with s the
// logistic function,
//   L_t = -c softplus(lam) s(r_t),  a_t = exp(L_t),  m_t = sqrt(1 - a_t^2),
//   h_t = a_t h_{t-1} + m_t s(i_t) x_t,   y = h.
// Gradients, with G_t = dy_t + a_{t+1} G_{t+1}:
//   dx = G m s(i),  di = G m x s(i) (1 - s(i)),
//   dL = G (a h_{t-1} - (a^2 / m) s(i) x),  dr = dL L (1 - s(r)),
//   dlam = sum_t dL L s(lam) / softplus(lam).
//
// A step h -> a h + b is a pair (a, b), and pairs compose, so time is cut into
// chunks of 128 rows, whatever sequences lie in them.  A workgroup takes one
// chunk of 64 or 128 channels, reads its rows once into registers (16 rows a
// wave), composes them, leaves the chunk's pair for the workgroups behind it,
// composes the pairs of the chunks in front, and applies the state that enters
// to its registers: every input is read once and every output written once.
//
// Forward, 8192 rows of 2048 bf16 channels in one sequence: 48.9 us with the kernel
// that prepares the words, 2.8 TB/s over what has to move (a copy: 5.1); the vector
// units are busy for 48%, and the wait for the chunks in front takes the rest.
// Gradients, 16384 rows of 4096 in 8 sequences: 262 us, 4.0 TB/s, vector units 73%
// busy; the forward call that leaves their states 136 us, 4.4 TB/s.
//
// The first row of a sequence does not look back: its pair is marked by a
// negative a (the decays are positive), and composing selects instead of
// multiplying, so that an infinity or a NaN stays in its own sequence.
#include "seq_common.h"

#include <type_traits>

namespace im2win {
namespace {

// Rows a wave holds in registers, by waves a workgroup: 16 x 8 rows take 59 us on the
// long prompt (before the gates took fewer instructions), 8 x 8 65, 8 x 16 and 16 x 4 67.
constexpr int kRows = 16;
// In the gradients, which hold twice as much of each: a training step 410 us, 444
// with 16 rows.
constexpr int kBwdRows = 8;
constexpr int kWaves = 8;
constexpr int kThreads = kWaves * kWave;
constexpr int kChunk = kRows * kWaves;    // rows of a workgroup
constexpr int kBwdChunk = kBwdRows * kWaves;
template <int R> constexpr uint32_t kAllRows = (1u << R) - 1;
// Chunks whose pairs are looked at one by one, behind the last whole group's state:
// the long prompt takes 50 us and a training step 410; with groups of 64 54 and 517.
constexpr int kGroup = 32;
constexpr int kLook = kGroup / kWaves;    // of those, the ones a wave looks at
constexpr float kReset = -1.0f;           // the a of a pair that does not look back
constexpr float kLog2e = 1.44269504088896f;

struct Pair {
    float a, b;
};

// first `p`, then `q`
__device__ __forceinline__ Pair then(Pair p, Pair q) {
    if (q.a < 0.0f) return q;
    return {p.a < 0.0f ? kReset : p.a * q.a, fmaf(q.a, p.b, q.b)};
}
__device__ __forceinline__ float apply(Pair q, float h) { return q.a < 0.0f ? q.b : fmaf(q.a, h, q.b); }

// ---------------------------------------------------------------------------
// Words that workgroups leave for each other: 64 bits in one access, so a word
// is whole or still the pattern that the fill kernel wrote.  No data beside
// the word is read, so relaxed accesses of the device's scope suffice.
// ---------------------------------------------------------------------------
constexpr uint64_t kEmpty = ~0ull;

__device__ __forceinline__ void leave(uint64_t* w, Pair p) {
    uint32_t a = __float_as_uint(p.a);
    if (a == 0xffffffffu) a = 0x7fc00000u;      // a NaN that would look like an empty word
    __hip_atomic_store(w, (uint64_t)__float_as_uint(p.b) << 32 | a, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ uint64_t look(const uint64_t* w) {
    return __hip_atomic_load(w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ Pair pair_of(uint64_t w) { return {__uint_as_float((uint32_t)w), __uint_as_float((uint32_t)(w >> 32))}; }

// 128-row chunks of a call, in the order of their tickets: a workgroup waits
// for chunks of smaller tickets only, and a ticket is drawn by a workgroup that
// runs, so every wait ends whatever order the workgroups start in.
struct Look {
    uint64_t* pairs;      // chunk x channel: the pair of a chunk's rows
    uint64_t* states;     // group x channel: the state behind a whole group (b of a pair)
    uint32_t* ticket;     // one less than the number of tickets drawn
    int chunks;
};


// ---------------------------------------------------------------------------
// The sequences' first and last rows inside of a chunk
// ---------------------------------------------------------------------------
template <int N>
struct Marks {
    int first[N];    // the sequence that begins at a row, or -1
    int last[N];     // the sequence that ends with a row, or -1
};

// Fills the marks of the chunk of rows [row0, row0 + N) and calls
// empty(b), with all lanes of a wave, for each sequence without rows that
// lies there (the last chunk: there or behind it).
template <int N, typename F>
__device__ __forceinline__ void mark(const SeqMap& seq, int row0, bool last_chunk, Marks<N>& m, F empty) {
    const int tid = threadIdx.x, lane = tid % kWave;
    if (!seq.starts) {
        if (tid < N) {
            const int t = row0 + tid;
            const bool in = t < seq.tokens;
            const int b = in ? t / seq.len : 0;
            m.first[tid] = in && t == b * seq.len ? b : -1;
            m.last[tid] = in && t + 1 == (b + 1) * seq.len ? b : -1;
        }
        __syncthreads();
        return;
    }
    if (tid < N) m.first[tid] = m.last[tid] = -1;
    __syncthreads();
    // sequences that begin in front of the chunk: all but the last of them end there
    const int skip = seq.before(row0);
    const int end = row0 + N;
    for (int base = (skip ? skip - 1 : 0) + tid / kWave * kWave; base < seq.count; base += kThreads) {
        const int b = base + lane;
        int f = 0, n = 0;
        bool mine = false;
        if (b < seq.count) {
            f = seq.clamped(b), n = seq.clamped(b + 1);
            mine = f < end || last_chunk;
            if (mine && n > f) {
                if (f >= row0 && f < end) m.first[f - row0] = b;
                if (n > row0 && n <= end) m.last[n - 1 - row0] = b;
            }
        }
        uint64_t none = __ballot(mine && n <= f && f >= row0);
        while (none) {
            const int k = __builtin_ctzll(none);
            none &= none - 1;
            empty(uniform(base + k));
        }
        if (!__ballot(mine)) break;
    }
    __syncthreads();
}

// The rows [t0, t0 + R) that lie in [lo, hi), a bit each
template <int R>
__device__ __forceinline__ uint32_t rows_inside(int t0, int lo, int hi) {
    const int from = lo - t0, to = hi - t0;
    const uint32_t upto = to <= 0 ? 0u : to >= R ? kAllRows<R> : (1u << to) - 1;
    return from <= 0 ? upto : from >= R ? 0u : upto & ~((1u << from) - 1);
}
// The rows of a wave that marks name, a bit each; the sequence itself is read where a bit is set.
template <int R>
__device__ __forceinline__ uint32_t marked(const int* m) {
    const int lane = threadIdx.x % kWave;
    return (uint32_t)__ballot(lane < R && m[lane % R] >= 0);
}

// ---------------------------------------------------------------------------
// V neighbouring channels of a row in a register: one element, or two bfloat16
// (4 bytes at any alignment).  Nothing beside the row is touched: the lane that
// would have an odd last channel takes the one before it too, and both lanes
// compute and write the same values there; lanes behind the row read what its
// last lane reads and write nothing.
// ---------------------------------------------------------------------------
template <typename T, int V>
struct Lane {
    int c;                    // first channel
    uint32_t offset, wide;    // its bytes in a row of T and of floats: 32 bits beside the row's scalar address
    bool on;
    __device__ __forceinline__ Lane(int first, int channels) {
        on = first < channels;
        c = first + V <= channels ? first : channels - V;
        offset = (uint32_t)c * (uint32_t)sizeof(T);
        wide = (uint32_t)c * 4u;
    }
    __device__ __forceinline__ uint32_t load(const T* row) const {
        if constexpr (V * sizeof(T) == 4) {
            uint32_t u;
            __builtin_memcpy(&u, reinterpret_cast<const char*>(row) + offset, 4);
            return u;
        } else {
            uint16_t u;
            __builtin_memcpy(&u, reinterpret_cast<const char*>(row) + offset, 2);
            return u;
        }
    }
    static __device__ __forceinline__ float get(uint32_t u, int v) {
        if constexpr (sizeof(T) == 4) return __uint_as_float(u);
        else return __uint_as_float(v ? u & 0xffff0000u : u << 16);
    }
    __device__ __forceinline__ void store(T* row, const float (&v)[V]) const {
        if (!on) return;
        char* p = reinterpret_cast<char*>(row) + offset;
        if constexpr (V == 1) {
            const T u = (T)v[0];
            __builtin_memcpy(p, &u, sizeof(T));
        } else {
            const uint32_t u = pack_bf16(v[0], v[1]);
            __builtin_memcpy(p, &u, 4);
        }
    }
    __device__ __forceinline__ void load(const float* row, float (&v)[V]) const { __builtin_memcpy(v, reinterpret_cast<const char*>(row) + wide, 4 * V); }
    __device__ __forceinline__ void store_f32(float* row, const float (&v)[V]) const {
        if (on) __builtin_memcpy(reinterpret_cast<char*>(row) + wide, v, 4 * V);
    }
};

// ---------------------------------------------------------------------------
// The gates of one element
// ---------------------------------------------------------------------------
struct Gate {
    float a, d;      // exp(L) and 1 - exp(2 L), for g = -L / ln 2 >= 0
};

// 1 - exp(2 L) loses all digits near L = 0, so where u = -2 L is below 0.25 it
// is the series u (1 - u/2! + u^2/3! - .. - u^5/6!), in powers of g = u / (2 ln
// 2) (its rest is under u^6 / 5040 = 5e-8); above, the subtraction is off by
// 9e-7 relative, and the root that is taken of it halves that.
__device__ __forceinline__ Gate gate_of(float g) {
    constexpr float k = 2.0f / kLog2e;
    constexpr float k1 = k, k2 = -k * k / 2, k3 = k * k * k / 6, k4 = -k * k * k * k / 24, k5 = k * k * k * k * k / 120, k6 = -k * k * k * k * k * k / 720;
    Gate o;
    o.a = __builtin_amdgcn_exp2f(-g);
    const float s = g * fmaf(g, fmaf(g, fmaf(g, fmaf(g, fmaf(g, k6, k5), k4), k3), k2), k1);
    o.d = g < 0.25f / k ? s : fmaf(-o.a, o.a, 1.0f);
    return o;
}

// c softplus(lam) log2(e): what s(r) is multiplied with
__device__ __forceinline__ float rate_of(float lam, float c) {
    const float sp = lam > 20.0f ? lam : log1pf(expf(lam));
    return c * sp * kLog2e;
}

// Empties the words that workgroups leave for each other, and works out the
// rates once (each workgroup on its own would add five instructions an element).
__global__ __launch_bounds__(256) void prepare_kernel(uint64_t* p, int64_t n, const float* lam, float* rates, int channels, float c) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i < n) p[i] = kEmpty;
    if (i < channels) rates[i] = rate_of(lam[i], c);
}

template <typename T, int V>
__device__ __forceinline__ void load_rates(const Lane<T, V>& own, const float* rates, const float* lam, float c, float (&r)[V]) {
    if (rates) {
        own.load(rates, r);
    } else {
        own.load(lam, r);
#pragma unroll
        for (int v = 0; v < V; ++v) r[v] = rate_of(r[v], c);
    }
}

struct RecArgs {
    const void *x, *r, *i;
    const float *lam, *rates;      // rates: NULL where one chunk holds all rows
    SeqMap seq;
    const float* init;
    void* y;              // NULL: only the states
    float* final_state;
    float* chunk_states;  // chunk of the gradients x channel, or NULL
    Look look;
    int64_t ld_x, ld_r, ld_i;
    int channels, tiles;
    float c;
};

// The state that enters a chunk: the state behind the group in front, then
// the pairs of the group's chunks in order, each wave composing kLook of them.
// `step` is +1 (time runs forwards) or -1; order counts chunks in that
// direction.  All threads of the workgroup take part; p holds V channels from c.
template <int V>
__device__ __forceinline__ void look_back(const Look& k, int order, int c, int channels, Pair (*pre)[kWave * V], float* enter, float (&h)[V]) {
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    const int group = order / kGroup, base = group * kGroup;
    Pair p[V];
#pragma unroll
    for (int v = 0; v < V; ++v) p[v] = {1.0f, 0.0f};
    const int from = base + wave * kLook;
    if (from < order) {
        uint64_t w[kLook][V];
        while (true) {
            bool ready = true;
#pragma unroll
            for (int j = 0; j < kLook; ++j) {
                const int q = from + j < order ? from + j : from;
#pragma unroll
                for (int v = 0; v < V; ++v) w[j][v] = look(k.pairs + (int64_t)q * channels + c + v);
            }
#pragma unroll
            for (int j = 0; j < kLook; ++j)
#pragma unroll
                for (int v = 0; v < V; ++v) ready &= w[j][v] != kEmpty;
            if (!__ballot(!ready)) break;
            __builtin_amdgcn_s_sleep(2);
        }
#pragma unroll
        for (int j = 0; j < kLook; ++j)
            if (from + j < order)
#pragma unroll
                for (int v = 0; v < V; ++v) p[v] = then(p[v], pair_of(w[j][v]));
    }
#pragma unroll
    for (int v = 0; v < V; ++v) pre[wave][lane * V + v] = p[v];
    if (wave == 0) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            uint64_t w = 0;
            if (group)
                while ((w = look(k.states + (int64_t)(group - 1) * channels + c + v)) == kEmpty) __builtin_amdgcn_s_sleep(2);
            enter[lane * V + v] = pair_of(w).b;
        }
    }
    __syncthreads();
#pragma unroll
    for (int v = 0; v < V; ++v) {
        h[v] = enter[lane * V + v];
        for (int w = 0; w < kWaves; ++w) h[v] = apply(pre[w][lane * V + v], h[v]);
    }
}

template <typename T, int V>
__global__ __launch_bounds__(kThreads, 2) void recurrence_kernel(RecArgs a) {
    __shared__ Marks<kChunk> marks;
    __shared__ Pair agg[kWaves][kWave * V];
    __shared__ Pair pre[kWaves][kWave * V];
    __shared__ float enter[kWave * V];
    __shared__ int drawn;
    const int wave = uniform(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    const bool many = a.look.chunks > 1;
    int ticket = blockIdx.x;
    if (many) {
        if (threadIdx.x == 0) drawn = (int)(atomicAdd(a.look.ticket, 1u) + 1u);
        __syncthreads();
        ticket = uniform(drawn);
    }
    const int chunk = ticket / a.tiles, tile = ticket - chunk * a.tiles;
    const int row0 = chunk * kChunk;
    const Lane<T, V> own((tile * kWave + lane) * V, a.channels);
    const int c = own.c;
    mark(a.seq, row0, chunk == a.look.chunks - 1, marks, [&](int b) {
        if (!a.final_state) return;
        float h[V] = {};
        if (a.init) own.load(a.init + (int64_t)b * a.channels, h);
        own.store_f32(a.final_state + (int64_t)b * a.channels, h);
    });
    const int lo = a.seq.first(0), hi = a.seq.first(a.seq.count);
    if (lo >= hi) return;      // of every workgroup: none waits

    const int t0 = row0 + wave * kRows;
    uint32_t xw[kRows], rw[kRows], iw[kRows];
    const int ts = t0 < lo ? lo : t0 >= hi ? hi - 1 : t0;
    const T* xp = static_cast<const T*>(a.x) + ts * a.ld_x;
    const T* rp = static_cast<const T*>(a.r) + ts * a.ld_r;
    const T* ip = static_cast<const T*>(a.i) + ts * a.ld_i;
#pragma unroll
    for (int j = 0; j < kRows; ++j) {
        xw[j] = own.load(xp);
        rw[j] = own.load(rp);
        iw[j] = own.load(ip);
        const bool on = t0 + j >= lo && t0 + j + 1 < hi;      // rows outside of the sequences are not read
        xp += on ? a.ld_x : 0;
        rp += on ? a.ld_r : 0;
        ip += on ? a.ld_i : 0;
    }
    float rate[V];
    load_rates(own, a.rates, a.lam, a.c, rate);

    float da[kRows][V], db[kRows][V];
    const uint32_t begin = marked<kRows>(marks.first + wave * kRows), end = marked<kRows>(marks.last + wave * kRows);
    const uint32_t inside = rows_inside<kRows>(t0, lo, hi);
#pragma unroll
    for (int j = 0; j < kRows; ++j)
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const Gate g = gate_of(rate[v] * sigmoid(own.get(rw[j], v)));
            da[j][v] = g.a;
            db[j][v] = __builtin_amdgcn_sqrtf(g.d) * sigmoid(own.get(iw[j], v)) * own.get(xw[j], v);
        }
    if (inside != kAllRows<kRows>) {
#pragma unroll
        for (int j = 0; j < kRows; ++j)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                da[j][v] = inside >> j & 1 ? da[j][v] : 1.0f;
                db[j][v] = inside >> j & 1 ? db[j][v] : 0.0f;
            }
    }
    // where sequences begin, their states from before are in b
    if (begin && a.init) {
#pragma unroll
        for (int j = 0; j < kRows; ++j) {
            if (!(begin >> j & 1)) continue;
            float h0[V];
            own.load(a.init + (int64_t)uniform(marks.first[wave * kRows + j]) * a.channels, h0);
#pragma unroll
            for (int v = 0; v < V; ++v) db[j][v] = fmaf(da[j][v], h0[v], db[j][v]);
        }
    }
    // the wave's rows as one pair; most waves hold no row that a sequence begins with
    Pair p[V];
    auto compose = [&](auto plain) {
#pragma unroll
        for (int v = 0; v < V; ++v) p[v] = {1.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < kRows; ++j) {
            const bool first = !plain && (begin >> j & 1);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                p[v].a *= da[j][v];
                p[v].b = first ? db[j][v] : fmaf(da[j][v], p[v].b, db[j][v]);
            }
        }
    };
    if (begin) compose(std::false_type{});
    else compose(std::true_type{});
#pragma unroll
    for (int v = 0; v < V; ++v) {
        if (begin) p[v].a = kReset;
        agg[wave][lane * V + v] = p[v];
    }
    __syncthreads();
    if (many && wave == 0 && chunk + 1 < a.look.chunks) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            Pair q = agg[0][lane * V + v];
            for (int w = 1; w < kWaves; ++w) q = then(q, agg[w][lane * V + v]);
            if (own.on) leave(a.look.pairs + (int64_t)chunk * a.channels + c + v, q);
        }
    }
    float h[V] = {};
    if (chunk) look_back<V>(a.look, chunk, c, a.channels, pre, enter, h);
    for (int w = 0; w < wave; ++w) {
#pragma unroll
        for (int v = 0; v < V; ++v) h[v] = apply(agg[w][lane * V + v], h[v]);
    }
    if (a.chunk_states && wave * kRows % kBwdChunk == 0 && t0 < a.seq.tokens) own.store_f32(a.chunk_states + (int64_t)(t0 / kBwdChunk) * a.channels, h);
    if (wave == kWaves - 1 && chunk % kGroup == kGroup - 1 && chunk + 1 < a.look.chunks) {
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (own.on) leave(a.look.states + (int64_t)(chunk / kGroup) * a.channels + c + v, {0.0f, apply(p[v], h[v])});
    }
    if (!a.y && !a.final_state) return;
    T* yp = static_cast<T*>(a.y) + (int64_t)t0 * a.channels;
    auto write = [&](auto plain) {
#pragma unroll
        for (int j = 0; j < kRows; ++j) {
            const bool first = !plain && (begin >> j & 1);
#pragma unroll
            for (int v = 0; v < V; ++v) h[v] = first ? db[j][v] : fmaf(da[j][v], h[v], db[j][v]);
            if (plain || ((inside >> j & 1) && a.y)) own.store(yp, h);
            yp += a.channels;
            if (!plain && (end >> j & 1) && a.final_state) own.store_f32(a.final_state + (int64_t)uniform(marks.last[wave * kRows + j]) * a.channels, h);
        }
    };
    if ((begin | end) || inside != kAllRows<kRows> || !a.y) write(std::false_type{});
    else write(std::true_type{});
}

// Final states (or gradients of initial ones) of sequences without rows when
// there are no rows at all: from[b], or zero.
__global__ __launch_bounds__(256) void copy_states_kernel(const float* from, float* to, int64_t n) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i < n) to[i] = from ? from[i] : 0.0f;
}

// ---------------------------------------------------------------------------
// Gradients: one pass too.  The state that enters a chunk comes from the
// forward call (chunk_states), the gradient that enters it from behind by the
// same look at the chunks behind it, e_t = a_t G_t in the place of h.
// ---------------------------------------------------------------------------
struct RecBwdArgs {
    const void *dy, *x, *r, *i;
    const float *lam, *rates;
    SeqMap seq;
    const float *init, *d_final, *chunk_states;
    void *dx, *dr, *di;
    float *d_init, *part;     // part: chunk x channel, the chunk's sum of dL L
    Look look;
    int64_t ld_x, ld_r, ld_i;
    int channels, tiles;
    float c;
};

template <typename T, int V>
__global__ __launch_bounds__(kThreads, 2) void recurrence_bwd_kernel(RecBwdArgs a) {
    __shared__ Marks<kBwdChunk> marks;
    __shared__ Pair agg[kWaves][kWave * V];
    __shared__ Pair back[kWaves][kWave * V];
    __shared__ Pair pre[kWaves][kWave * V];
    __shared__ float enter[kWave * V];
    __shared__ int drawn;
    const int wave = uniform(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    const bool many = a.look.chunks > 1;
    int ticket = blockIdx.x;
    if (many) {
        if (threadIdx.x == 0) drawn = (int)(atomicAdd(a.look.ticket, 1u) + 1u);
        __syncthreads();
        ticket = uniform(drawn);
    }
    const int order = ticket / a.tiles, tile = ticket - order * a.tiles;
    const int chunk = a.look.chunks - 1 - order;
    const int row0 = chunk * kBwdChunk;
    const Lane<T, V> own((tile * kWave + lane) * V, a.channels);
    const int c = own.c;
    mark(a.seq, row0, order == 0, marks, [&](int b) {
        if (!a.d_init) return;
        float h[V] = {};
        if (a.d_final) own.load(a.d_final + (int64_t)b * a.channels, h);
        own.store_f32(a.d_init + (int64_t)b * a.channels, h);
    });
    const int lo = a.seq.first(0), hi = a.seq.first(a.seq.count);
    if (lo >= hi) {            // of every workgroup: none waits
        const float zero[V] = {};
        if (wave == 0) own.store_f32(a.part + (int64_t)chunk * a.channels, zero);
        return;
    }

    const int t0 = row0 + wave * kBwdRows;
    uint32_t xw[kBwdRows], rw[kBwdRows], iw[kBwdRows], gw[kBwdRows];
    const int ts = t0 < lo ? lo : t0 >= hi ? hi - 1 : t0;
    const T* xp = static_cast<const T*>(a.x) + ts * a.ld_x;
    const T* rp = static_cast<const T*>(a.r) + ts * a.ld_r;
    const T* dp = static_cast<const T*>(a.dy) + (int64_t)ts * a.channels;
    const T* ip = static_cast<const T*>(a.i) + ts * a.ld_i;
#pragma unroll
    for (int j = 0; j < kBwdRows; ++j) {
        xw[j] = own.load(xp);
        rw[j] = own.load(rp);
        iw[j] = own.load(ip);
        gw[j] = own.load(dp);
        const bool on = t0 + j >= lo && t0 + j + 1 < hi;      // rows outside of the sequences are not read
        xp += on ? a.ld_x : 0;
        rp += on ? a.ld_r : 0;
        ip += on ? a.ld_i : 0;
        dp += on ? a.channels : 0;
    }
    float rate[V], h[V] = {};
    load_rates(own, a.rates, a.lam, a.c, rate);
    if (chunk) own.load(a.chunk_states + (int64_t)chunk * a.channels, h);

    // hb: first the row's b, then the state in front of the row
    float da[kBwdRows][V], hb[kBwdRows][V];
    const uint32_t begin = marked<kBwdRows>(marks.first + wave * kBwdRows), end = marked<kBwdRows>(marks.last + wave * kBwdRows);
    const uint32_t inside = rows_inside<kBwdRows>(t0, lo, hi);
#pragma unroll
    for (int j = 0; j < kBwdRows; ++j)
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const Gate g = gate_of(rate[v] * sigmoid(own.get(rw[j], v)));
            da[j][v] = g.a;
            hb[j][v] = __builtin_amdgcn_sqrtf(g.d) * sigmoid(own.get(iw[j], v)) * own.get(xw[j], v);
        }
    if (inside != kAllRows<kBwdRows>) {
#pragma unroll
        for (int j = 0; j < kBwdRows; ++j) {
            if (!(inside >> j & 1)) gw[j] = 0;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                da[j][v] = inside >> j & 1 ? da[j][v] : 1.0f;
                hb[j][v] = inside >> j & 1 ? hb[j][v] : 0.0f;
            }
        }
    }
    auto initial = [&](int j, float (&h0)[V]) {
#pragma unroll
        for (int v = 0; v < V; ++v) h0[v] = 0.0f;
        if (a.init) own.load(a.init + (int64_t)uniform(marks.first[wave * kBwdRows + j]) * a.channels, h0);
    };
    auto after = [&](int j, float (&g0)[V]) {
#pragma unroll
        for (int v = 0; v < V; ++v) g0[v] = 0.0f;
        if (a.d_final) own.load(a.d_final + (int64_t)uniform(marks.last[wave * kBwdRows + j]) * a.channels, g0);
    };
    Pair p[V], q[V];
    auto compose = [&](auto plain) {
#pragma unroll
        for (int v = 0; v < V; ++v) p[v] = q[v] = {1.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < kBwdRows; ++j) {
            if (!plain && (begin >> j & 1)) {
                float h0[V];
                initial(j, h0);
#pragma unroll
                for (int v = 0; v < V; ++v) p[v].b = h0[v];
            }
#pragma unroll
            for (int v = 0; v < V; ++v) {
                p[v].a *= da[j][v];
                p[v].b = fmaf(da[j][v], p[v].b, hb[j][v]);
            }
        }
#pragma unroll
        for (int j = kBwdRows - 1; j >= 0; --j) {
            if (!plain && (end >> j & 1)) {
                float g0[V];
                after(j, g0);
#pragma unroll
                for (int v = 0; v < V; ++v) q[v].b = g0[v];
            }
#pragma unroll
            for (int v = 0; v < V; ++v) q[v].b = da[j][v] * (q[v].b + own.get(gw[j], v));
        }
#pragma unroll
        for (int v = 0; v < V; ++v) q[v].a = p[v].a;      // the same product
    };
    if (begin | end) compose(std::false_type{});
    else compose(std::true_type{});
#pragma unroll
    for (int v = 0; v < V; ++v) {
        if (begin) p[v].a = kReset;
        if (end) q[v].a = kReset;
        agg[wave][lane * V + v] = p[v];
        back[wave][lane * V + v] = q[v];
    }
    __syncthreads();
    if (many && wave == 0 && chunk) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            Pair s = back[kWaves - 1][lane * V + v];
            for (int w = kWaves - 2; w >= 0; --w) s = then(s, back[w][lane * V + v]);
            if (own.on) leave(a.look.pairs + (int64_t)order * a.channels + c + v, s);
        }
    }
    for (int w = 0; w < wave; ++w) {
#pragma unroll
        for (int v = 0; v < V; ++v) h[v] = apply(agg[w][lane * V + v], h[v]);
    }
    auto states = [&](auto plain) {
#pragma unroll
        for (int j = 0; j < kBwdRows; ++j) {
            if (!plain && (begin >> j & 1)) initial(j, h);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float before = h[v];
                h[v] = fmaf(da[j][v], h[v], hb[j][v]);
                hb[j][v] = before;
            }
        }
    };
    if (begin) states(std::false_type{});
    else states(std::true_type{});
    float g[V] = {};
    if (order) look_back<V>(a.look, order, c, a.channels, pre, enter, g);
    for (int w = kWaves - 1; w > wave; --w) {
#pragma unroll
        for (int v = 0; v < V; ++v) g[v] = apply(back[w][lane * V + v], g[v]);
    }
    if (wave == 0 && order % kGroup == kGroup - 1 && chunk) {
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (own.on) leave(a.look.states + (int64_t)(order / kGroup) * a.channels + c + v, {0.0f, apply(q[v], g[v])});
    }
    float sum[V] = {};
    const int64_t behind = (int64_t)(t0 + kBwdRows) * a.channels;
    T *dx = static_cast<T*>(a.dx) + behind, *dr = static_cast<T*>(a.dr) + behind, *di = static_cast<T*>(a.di) + behind;
    auto write = [&](auto plain) {
#pragma unroll
        for (int j = kBwdRows - 1; j >= 0; --j) {
            dx -= a.channels;
            dr -= a.channels;
            di -= a.channels;
            if (!plain && !(inside >> j & 1)) continue;
            if (!plain && (end >> j & 1)) after(j, g);
            // the gates again: kept from above, they would take four registers an element
            arrive(rw[j]);
            arrive(iw[j]);
            float ox[V], orr[V], oi[V];
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float x = own.get(xw[j], v), sr = sigmoid(own.get(rw[j], v)), si = sigmoid(own.get(iw[j], v));
                const float gg = g[v] + own.get(gw[j], v);
                const float l2 = rate[v] * sr;                   // -L / ln 2
                const Gate gt = gate_of(l2);
                // 1 / m; L / m goes to zero with L, and is zero where both are
                const float d = fmaxf(gt.d, 0x1p-125f), im = __builtin_amdgcn_rsqf(d);
                const float l = l2 * (-1.0f / kLog2e), gm = gg * (d * im);
                const float dl = gg * gt.a * fmaf(-gt.a * (l * im), si * x, l * hb[j][v]);      // dL L
                ox[v] = gm * si;
                oi[v] = ox[v] * fmaf(-si, x, x);
                orr[v] = fmaf(-sr, dl, dl);
                sum[v] += dl;
                g[v] = gt.a * gg;
            }
            own.store(dx, ox);
            own.store(dr, orr);
            own.store(di, oi);
            if (!plain && (begin >> j & 1) && a.d_init) own.store_f32(a.d_init + (int64_t)uniform(marks.first[wave * kBwdRows + j]) * a.channels, g);
            __builtin_amdgcn_sched_barrier(0);      // a row at a time: mixed, the rows' temporaries spill
        }
    };
    if ((begin | end) || inside != kAllRows<kBwdRows>) write(std::false_type{});
    else write(std::true_type{});
    __syncthreads();
#pragma unroll
    for (int v = 0; v < V; ++v) pre[wave][lane * V + v].b = sum[v];
    __syncthreads();
    if (wave == 0) {
#pragma unroll
        for (int v = 0; v < V; ++v)
            for (int w = 1; w < kWaves; ++w) sum[v] += pre[w][lane * V + v].b;
        own.store_f32(a.part + (int64_t)chunk * a.channels, sum);
    }
}

// dlam from the chunks' sums: 64 channels a workgroup, every 16th chunk a wave
constexpr int kSumWaves = 16;
__global__ __launch_bounds__(kSumWaves * kWave) void recurrence_bwd_sum_kernel(const float* part, const float* lam, float* dlam, int chunks, int channels) {
    __shared__ float sum[kSumWaves][kWave];
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    const int c = (int)blockIdx.x * kWave + lane;
    float s = 0.0f;
    if (c < channels) {
#pragma unroll 8
        for (int i = wave; i < chunks; i += kSumWaves) s += part[(int64_t)i * channels + c];
    }
    sum[wave][lane] = s;
    __syncthreads();
    if (wave == 0 && c < channels) {
        for (int i = 1; i < kSumWaves; ++i) s += sum[i][lane];
        // s(lam) / softplus(lam): with e = exp(lam), e / ((1 + e) log1p(e)), which goes to 1 with e
        const float l = lam[c], e = expf(l);
        const float ratio = l > 20.0f ? 1.0f / l : e > 0.0f ? e / ((1.0f + e) * log1pf(e)) : 1.0f;
        dlam[c] = s * ratio;
    }
}

// ---------------------------------------------------------------------------
// One token of each request
// ---------------------------------------------------------------------------
struct RecStepArgs {
    const void *x, *r, *i;
    const float* lam;
    const int32_t* slots;
    float* state;
    void* y;
    int64_t ld_x, ld_r, ld_i, state_slots;
    int channels;
    float c;
};

template <typename T, int V>
__global__ __launch_bounds__(256) void recurrence_step_kernel(RecStepArgs a) {
    const int c = ((int)blockIdx.y * 256 + (int)threadIdx.x) * V, n = a.channels - c;
    if (n <= 0) return;
    const int64_t t = blockIdx.x;
    const int64_t slot = a.slots ? a.slots[t] : t;
    const bool live = slot >= 0 && slot < a.state_slots;
    float* st = a.state + (live ? slot : 0) * a.channels + c;
    const T* x = static_cast<const T*>(a.x) + t * a.ld_x + c;
    const T* r = static_cast<const T*>(a.r) + t * a.ld_r + c;
    const T* i = static_cast<const T*>(a.i) + t * a.ld_i + c;
    T* y = static_cast<T*>(a.y) + t * a.channels + c;
    // (the scans' lanes share an odd last channel; here each has its own, since the state moves in place)
#pragma unroll
    for (int v = 0; v < V; ++v) {
        if (v >= n) continue;
        if (!live) {
            y[v] = (T)0.0f;
            continue;
        }
        const Gate g = gate_of(rate_of(a.lam[c + v], a.c) * sigmoid((float)r[v]));
        const float h = fmaf(g.a, st[v], __builtin_amdgcn_sqrtf(g.d) * sigmoid((float)i[v]) * (float)x[v]);
        y[v] = (T)h;
        st[v] = h;
    }
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
int check_desc(const im2win_recurrence_desc* d) {
    if (!d) return fail(IM2WIN_ENULL, "descriptor is NULL");
    int rc = check_rows(d->tokens, d->channels, d->dtype);
    if (rc) return rc;
    if (!(d->c > 0.0f) || d->c > 1e30f) return fail(IM2WIN_EINVAL, "c must be positive (got %g)", (double)d->c);
    if ((rc = check_ld(d->ld_x, d->channels, "ld_x")) || (rc = check_ld(d->ld_r, d->channels, "ld_r")) || (rc = check_ld(d->ld_i, d->channels, "ld_i"))) return rc;
    return IM2WIN_OK;
}

// Channels of a lane: 4 bytes of a row, or a row of one bfloat16
int lane_channels(const im2win_recurrence_desc* d) { return d->dtype == IM2WIN_F32 || d->channels == 1 ? 1 : 2; }

struct Plan {
    int64_t chunks, tiles;
    size_t words, look_bytes, states_bytes, total;
};

Plan plan_of(const im2win_recurrence_desc* d, int chunk) {
    Plan p{};
    p.chunks = (d->tokens + chunk - 1) / chunk;
    const int64_t per = kWave * lane_channels(d);
    p.tiles = (d->channels + per - 1) / per;
    if (p.chunks > 1) p.words = (size_t)((p.chunks + p.chunks / kGroup) * d->channels + 2);      // pairs, states, ticket, to 16 bytes
    p.look_bytes = p.words ? (p.words * 8 + 15) / 16 * 16 + ((size_t)d->channels * 4 + 15) / 16 * 16 : 0;      // the rates behind the words
    p.states_bytes = ((size_t)(p.chunks * d->channels) * 4 + 15) / 16 * 16;
    return p;
}

int check_plan(const im2win_recurrence_desc* d, const Plan& p) {
    int rc = check_launch(p.chunks * p.tiles, kThreads, "gated_recurrence");
    if (!rc) rc = check_launch(((int64_t)p.words + 255) / 256, 256, "gated_recurrence's workspace");
    if (!rc && d->tokens == 0) rc = check_launch((d->sequences * d->channels + 255) / 256, 256, "gated_recurrence's states");
    return rc;
}

Look look_of(const Plan& p, int64_t channels, void* ws) {
    Look k{};
    k.chunks = (int)p.chunks;
    if (p.chunks > 1) {
        k.ticket = static_cast<uint32_t*>(ws);
        k.pairs = static_cast<uint64_t*>(ws) + 2;
        k.states = k.pairs + p.chunks * channels;
    }
    return k;
}

// Empties the words and works out the rates; where they lie, or NULL.
const float* prepare(const im2win_recurrence_desc* d, const Plan& p, const float* lam, void* ws, hipStream_t s) {
    if (!p.words) return nullptr;
    float* rates = reinterpret_cast<float*>(static_cast<char*>(ws) + (p.words * 8 + 15) / 16 * 16);
    // there are at least as many words as channels
    hipLaunchKernelGGL(prepare_kernel, dim3((unsigned)((p.words + 255) / 256)), dim3(256), 0, s, static_cast<uint64_t*>(ws), (int64_t)p.words, lam, rates,
                       (int)d->channels, d->c);
    return rates;
}

template <typename F>
void with_type(const im2win_recurrence_desc* d, F f) {
    using std::integral_constant;
    if (d->dtype == IM2WIN_F32) f(float{}, integral_constant<int, 1>{});
    else if (lane_channels(d) == 1) f(bf16{}, integral_constant<int, 1>{});
    else f(bf16{}, integral_constant<int, 2>{});
}

int launch_forward(const im2win_recurrence_desc* d, const Plan& p, RecArgs& a, void* ws, hipStream_t s) {
    a.look = look_of(p, d->channels, ws);
    a.ld_x = d->ld_x; a.ld_r = d->ld_r; a.ld_i = d->ld_i;
    a.channels = (int)d->channels; a.tiles = (int)p.tiles; a.c = d->c;
    a.rates = prepare(d, p, a.lam, ws, s);
    with_type(d, [&](auto t, auto v) {
        hipLaunchKernelGGL((recurrence_kernel<decltype(t), decltype(v)::value>), dim3((unsigned)(p.chunks * p.tiles)), dim3(kThreads), 0, s, a);
    });
    return launched("gated_recurrence");
}

int copy_states(const float* from, float* to, int64_t n, hipStream_t s) {
    if (to && n) hipLaunchKernelGGL(copy_states_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, from, to, n);
    return launched("gated_recurrence's states");
}

}  // namespace
}  // namespace im2win

using namespace im2win;

extern "C" {

int im2win_gated_recurrence_chunks(const im2win_recurrence_desc* d, int64_t* chunks) {
    int rc = check_desc(d);
    if (rc) return rc;
    if (!chunks) return fail(IM2WIN_ENULL, "chunks is NULL");
    *chunks = plan_of(d, kBwdChunk).chunks;
    return ok();
}

int im2win_gated_recurrence_workspace_bytes(const im2win_recurrence_desc* d, size_t* bytes) {
    int rc = check_desc(d);
    if (rc) return rc;
    if (!bytes) return fail(IM2WIN_ENULL, "bytes is NULL");
    *bytes = plan_of(d, kChunk).look_bytes;
    return ok();
}

int im2win_gated_recurrence(const im2win_recurrence_desc* d, const void* x, const void* r, const void* i, const float* lam,
                            const int32_t* seq_starts, const float* initial_state, void* y, float* final_state,
                            float* chunk_states, void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_desc(d);
    if (rc || (rc = check_sequences(d->tokens, d->sequences, seq_starts, true)) || (rc = need_ptr(lam, 4, "lam")) ||
        (rc = may_ptr(initial_state, 4, "initial_state")) || (rc = may_ptr(final_state, 4, "final_state")) ||
        (rc = may_ptr(chunk_states, 4, "chunk_states")))
        return rc;
    const Plan p = plan_of(d, kChunk);
    const size_t e = size_of(d->dtype);
    if (d->tokens && ((rc = need_ptr(x, e, "x")) || (rc = need_ptr(r, e, "r")) || (rc = need_ptr(i, e, "i")) || (rc = need_ptr(y, e, "y")))) return rc;
    if (p.look_bytes && (rc = need_ptr(workspace, 16, "workspace"))) return rc;
    if (workspace_bytes < p.look_bytes)
        return fail(IM2WIN_EWORKSPACE, "workspace holds %zu bytes, the recurrence needs %zu", workspace_bytes, p.look_bytes);
    if ((rc = check_plan(d, p))) return rc;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (d->tokens == 0) return copy_states(initial_state, final_state, d->sequences * d->channels, s);
    RecArgs a{};
    a.x = x; a.r = r; a.i = i; a.lam = lam; a.seq = make_seq_map(d->tokens, d->sequences, seq_starts);
    a.init = initial_state; a.y = y; a.final_state = final_state; a.chunk_states = chunk_states;
    return launch_forward(d, p, a, workspace, s);
}

int im2win_gated_recurrence_backward_workspace_bytes(const im2win_recurrence_desc* d, size_t* bytes) {
    int rc = check_desc(d);
    if (rc) return rc;
    if (!bytes) return fail(IM2WIN_ENULL, "bytes is NULL");
    const Plan p = plan_of(d, kBwdChunk);
    *bytes = p.look_bytes + 2 * p.states_bytes;     // the look, the chunks' sums, the chunks' states
    return ok();
}

int im2win_gated_recurrence_backward(const im2win_recurrence_desc* d, const void* dy, const void* x, const void* r, const void* i,
                                     const float* lam, const int32_t* seq_starts, const float* initial_state,
                                     const float* d_final_state, const float* chunk_states, void* dx, void* dr, void* di,
                                     float* dlam, float* d_initial_state, void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_desc(d);
    if (rc || (rc = check_sequences(d->tokens, d->sequences, seq_starts, true)) || (rc = need_ptr(lam, 4, "lam")) ||
        (rc = need_ptr(dlam, 4, "dlam")) || (rc = may_ptr(initial_state, 4, "initial_state")) ||
        (rc = may_ptr(d_final_state, 4, "d_final_state")) || (rc = may_ptr(d_initial_state, 4, "d_initial_state")) ||
        (rc = may_ptr(chunk_states, 4, "chunk_states")))
        return rc;
    const Plan p = plan_of(d, kBwdChunk);
    const size_t e = size_of(d->dtype), need = p.look_bytes + 2 * p.states_bytes;
    if (d->tokens && ((rc = need_ptr(dy, e, "dy")) || (rc = need_ptr(x, e, "x")) || (rc = need_ptr(r, e, "r")) || (rc = need_ptr(i, e, "i")) ||
                      (rc = need_ptr(dx, e, "dx")) || (rc = need_ptr(dr, e, "dr")) || (rc = need_ptr(di, e, "di")) ||
                      (rc = need_ptr(workspace, 16, "workspace"))))
        return rc;
    if (workspace_bytes < need)
        return fail(IM2WIN_EWORKSPACE, "workspace holds %zu bytes, the gradients need %zu", workspace_bytes, need);
    if ((rc = check_plan(d, p))) return rc;
    hipStream_t s = static_cast<hipStream_t>(stream);
    char* ws = static_cast<char*>(workspace);
    float* part = reinterpret_cast<float*>(ws + p.look_bytes);
    if (d->tokens) {
        const SeqMap seq = make_seq_map(d->tokens, d->sequences, seq_starts);
        if (!chunk_states && p.chunks > 1) {
            RecArgs f{};
            f.x = x; f.r = r; f.i = i; f.lam = lam; f.seq = seq; f.init = initial_state;
            f.chunk_states = reinterpret_cast<float*>(ws + p.look_bytes + p.states_bytes);
            chunk_states = f.chunk_states;
            if ((rc = launch_forward(d, plan_of(d, kChunk), f, ws, s))) return rc;      // of fewer chunks: its words fit where the gradients' lie
        }
        RecBwdArgs a{};
        a.dy = dy; a.x = x; a.r = r; a.i = i; a.lam = lam; a.seq = seq;
        a.init = initial_state; a.d_final = d_final_state; a.chunk_states = chunk_states;
        a.dx = dx; a.dr = dr; a.di = di; a.d_init = d_initial_state; a.part = part;
        a.look = look_of(p, d->channels, ws);
        a.ld_x = d->ld_x; a.ld_r = d->ld_r; a.ld_i = d->ld_i;
        a.channels = (int)d->channels; a.tiles = (int)p.tiles; a.c = d->c;
        a.rates = prepare(d, p, lam, ws, s);
        with_type(d, [&](auto t, auto v) {
            hipLaunchKernelGGL((recurrence_bwd_kernel<decltype(t), decltype(v)::value>), dim3((unsigned)(p.chunks * p.tiles)), dim3(kThreads), 0, s, a);
        });
    } else if ((rc = copy_states(d_final_state, d_initial_state, d->sequences * d->channels, s))) {
        return rc;
    }
    hipLaunchKernelGGL(recurrence_bwd_sum_kernel, dim3((unsigned)((d->channels + kWave - 1) / kWave)), dim3(kSumWaves * kWave), 0, s,
                       part, lam, dlam, (int)p.chunks, (int)d->channels);
    return launched("gated_recurrence_backward");
}

int im2win_gated_recurrence_step(const im2win_recurrence_desc* d, const void* x, const void* r, const void* i, const float* lam,
                                 const int32_t* slots, float* state, int64_t state_slots, void* y, void* stream) {
    int rc = check_desc(d);
    if (rc || (rc = need_ptr(lam, 4, "lam"))) return rc;
    if (state_slots < 0) return fail(IM2WIN_EINVAL, "state_slots must be >= 0 (got %lld)", (long long)state_slots);
    if (d->tokens == 0) return ok();
    const size_t e = size_of(d->dtype);
    if ((rc = need_ptr(x, e, "x")) || (rc = need_ptr(r, e, "r")) || (rc = need_ptr(i, e, "i")) || (rc = need_ptr(y, e, "y")) ||
        (rc = may_ptr(slots, 4, "slots")) || (rc = need_ptr(state, 4, "state")))
        return rc;
    const int64_t per = 256 * lane_channels(d), tiles = (d->channels + per - 1) / per;
    if ((rc = check_launch(d->tokens * tiles, 256, "gated_recurrence_step"))) return rc;
    RecStepArgs a{};
    a.x = x; a.r = r; a.i = i; a.lam = lam; a.slots = slots; a.state = state; a.y = y;
    a.ld_x = d->ld_x; a.ld_r = d->ld_r; a.ld_i = d->ld_i; a.state_slots = state_slots;
    a.channels = (int)d->channels; a.c = d->c;
    with_type(d, [&](auto t, auto v) {
        hipLaunchKernelGGL((recurrence_step_kernel<decltype(t), decltype(v)::value>), dim3((unsigned)d->tokens, (unsigned)tiles), dim3(256), 0, static_cast<hipStream_t>(stream), a);
    });
    return launched("gated_recurrence_step");
}

}  // extern "C"
