// Gradients of the selective scan (im2win_selective_scan_backward,
// include/im2win_seq.h).
//
// With s the step size, a = exp(s A), u = s x and p = dy silu(z) the gradient
// of the sum in front of the gate, the gradient g_t of the state h_t obeys
//   g_t = C_t p_t + a_{t+1} g_{t+1}          (along a sequence, from its end),
// and   dC_t = sum_c p h,        dB_t = sum_c g u   (over the group's channels),
//       q_t  = g a h_{t-1},      dA = sum_t q s,
//       du   = sum_n g B,        dx = du s + D p,   ds = du x + sum_n q A.
// Chunks of rows as in the forward scan, in four kernels:
//   1. each chunk's state from zero and, in the same walk, the gradient that
//      its rows send to the state before it: sum_t (prod_{r<=t} a_r) C_t p_t;
//   2. both carried over the chunks, forwards and backwards (left to kernel 3
//      where sequences are few chunks long);
//   3. each chunk: a walk forwards that leaves the state before every tile of
//      rows in LDS, then the tiles from the last to the first: the tile's
//      states again into registers, then its rows backwards;
//   4. the sums over chunks (dA, dD, ddt_bias) and over workgroups (dB, dC).
// The sums over channels of dB and dC run over a wave's 16 quads: four values
// at a time fold into one register by swapping halves and rows of lanes, so
// that a value costs two instructions instead of four exchanges.
//
// Bound by issue slots: per row, channel and state kernel 1 takes eight, the
// walk forwards of kernel 3 five, the states again five, the row backwards
// twelve and the folds two.  8 x 2048 rows of 2048 x 16 bf16 take 770 us; under
// the profiler 173 in kernel 1, 46 in 2, 557 in 3 (90% of its slots taken), 28 in
// 4; chunks of 64 rows write and read 0.3 GB of states, shorter ones more.
#include <algorithm>

#include "seq_scan.h"

namespace im2win {
namespace {

struct ScanBwdArgs {
    ScanArgs s;
    const void* dy;
    const float* d_final;
    void* dx;
    void* ddt;
    float* dA;
    void* dB;
    void* dC;
    float* dD;
    void* dz;
    float* ddt_bias;
    float* d_init;
    float* back;      // [chunks][channels][4*NS]: the gradient of the state before each chunk
    float* dbc;       // [group_blocks][tokens][G][2][4*NS]
    float* da_part;   // [chunks][channels][4*NS]
    float* dd_part;   // [chunks][channels][2]: dD and ddt_bias
    int groups;
};

// Rows of a tile whose states are in registers, and of a chunk (whose tiles'
// first states, B and C lie in LDS)
template <int NS> constexpr int kTileRows = NS >= 16 || NS == 6 ? 4 : 8;
template <int NS> constexpr int kChunkRows = NS == 32 ? 12 : NS == 16 || NS == 6 ? 24 : 64;

template <int NS, int CH>
struct BwdLds {
    static constexpr int NP = kQuad * NS, Q = kChunkRows<NS>, TB = kTileRows<NS>;
    float b[Q * NP], c[Q * NP];
    float part[kScanWaves][TB][2 * NP];
    float state[kScanWaves][Q / TB][CH * NS][kWave];
};

// The chunk's rows and the sequence of one of them
struct ChunkRows {
    int lo, hi;
    __device__ __forceinline__ ChunkRows(const ScanArgs& a, int chunk) {
        lo = max(a.seq.first(0), chunk * a.chunk);
        hi = min(a.seq.first(a.seq.count), min(chunk * a.chunk, a.seq.tokens - a.chunk) + a.chunk);
    }
};

// A state of sequence b (zero where m is NULL).  Places that are not live hold zeros throughout,
// so that they add nothing to sums over channels.
template <int NS, int CH>
__device__ __forceinline__ void load_state(const float* m, const ScanArgs& a, const Lane<CH>& l, int b, float (&h)[CH][NS]) {
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        if (m) load_states<NS>(m + ((int64_t)b * a.channels + l.c + i) * a.states, l.q, a.states, h[i]);
#pragma unroll
        for (int s = 0; s < NS; ++s) h[i][s] = m && l.live[i] ? h[i][s] : 0.0f;
    }
}

template <int NS, int CH>
__device__ __forceinline__ void load_decay(const ScanArgs& a, const Lane<CH>& l, float (&a2)[CH][NS]) {
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        load_states<NS>(a.A + (int64_t)(l.c + i) * a.states, l.q, a.states, a2[i]);
#pragma unroll
        for (int s = 0; s < NS; ++s) a2[i][s] = l.live[i] ? kLog2e * a2[i][s] : 0.0f;
    }
}

// What four rows (one per lane of the quad) need in the walks
template <typename T, int CH>
struct BwdRows {
    Raw<T, CH> x, dt, z, dy;

    __device__ __forceinline__ void wait() {
        x.wait();
        dt.wait();
        z.wait();
        dy.wait();
    }
    __device__ __forceinline__ float step(const ScanArgs& a, int i, float bias) const {
        const float v = dt.get(i) + bias;
        return a.softplus ? softplus(v) : v;
    }
    // the gradient of the sum in front of the gate
    __device__ __forceinline__ float grad(const ScanArgs& a, int i) const {
        const float g = dy.get(i);
        if (!a.z) return g;
        const float v = z.get(i);
        return g * v * sigmoid(v);
    }
};
template <typename T, int CH>
struct BwdPlaces {
    RowPlace<T> x, dt, z, dense;
    __device__ __forceinline__ BwdPlaces(const ScanArgs& a, const Lane<CH>& l, int row)
        : x(a.ld_x, l, row), dt(a.ld_dt, l, row), z(a.ld_z, l, row), dense(a.channels, l, row) {}
    __device__ __forceinline__ void load_in(const ScanArgs& a, int t, BwdRows<T, CH>& r) const {
        r.x.load(x.at(a.x, a.ld_x, t));
        r.dt.load(dt.at(a.dt, a.ld_dt, t));
    }
    __device__ __forceinline__ void load_grad(const ScanBwdArgs& p, int t, BwdRows<T, CH>& r) const {
        if (p.s.z) r.z.load(z.at(p.s.z, p.s.ld_z, t));
        r.dy.load(dense.at(p.dy, p.s.channels, t));
    }
};

// ---------------------------------------------------------------------------
// 1. What a chunk does to the states: forwards for its last sequence, where
// that goes on, and backwards for its first, where that began before.
// ---------------------------------------------------------------------------
template <typename T, int NS, int CH>
__global__ __launch_bounds__(kScanWaves * kWave) void scan_bwd_summary_kernel(ScanBwdArgs p) {
    constexpr int NP = kQuad * NS;
    const ScanArgs& a = p.s;
    __shared__ __align__(16) float sb[kScanTile * NP];
    __shared__ __align__(16) float sc[kScanTile * NP];
    const int block = blockIdx.x % a.blocks, chunk = blockIdx.x / a.blocks;
    const int wave = uniform(threadIdx.x / kWave);
    const ChunkRows rows(a, chunk);
    int flags = 0, b0 = 0, end0 = 0, b1 = 0, first1 = 0;
    if (rows.lo < rows.hi) {
        const SeqMap::Found f0 = a.seq.at(rows.lo), f1 = a.seq.at(rows.hi - 1);
        b0 = f0.b;
        b1 = f1.b;
        end0 = f0.end;
        first1 = f1.first;
        const int first0 = f0.first, end1 = f1.end;
        flags = (end1 > rows.hi ? kGoesOn : 0) | (first0 < rows.lo ? kFromBefore : 0);
        if (first0 < rows.lo && end0 > rows.hi) flags |= kThrough;
    }
    if (block == 0 && threadIdx.x == 0) a.flags[chunk] = flags;
    if (!(flags & (kGoesOn | kFromBefore))) return;

    Lane<CH> l;
    l.init(a, block, wave);
    const int group_offset = block / a.group_blocks * a.states;
    float a2[CH][NS], bias[CH];
    load_decay<NS, CH>(a, l, a2);
#pragma unroll
    for (int i = 0; i < CH; ++i) bias[i] = a.dt_bias ? a.dt_bias[l.c + i] : 0.0f;

    // rows [from, to) of one sequence: h from its value before, the sum of steps, and the gradient sent back
    float h[CH][NS], back[CH][NS], pass[CH][NS], span[CH];
    auto walk = [&](int from, int to) {
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            span[i] = 0.0f;
#pragma unroll
            for (int s = 0; s < NS; ++s) {
                back[i][s] = 0.0f;
                pass[i][s] = 1.0f;
            }
        }
        BwdPlaces<T, CH> places(a, l, l.q);
        auto load = [&](int t, BwdRows<T, CH>& r) {
            if (t + kQuad > to) places = BwdPlaces<T, CH>(a, l, min(l.q, to - 1 - t));     // the last group
            places.load_in(a, t, r);
            places.load_grad(p, t, r);
        };
        BwdRows<T, CH> next;
        load(from, next);
        for (int tile = from; tile < to; tile += kScanTile) {
            const int n = min(kScanTile, to - tile);
            __syncthreads();
            stage<T, NS>(sb, static_cast<const T*>(a.B), a.ld_b, group_offset, a.states, tile, n);
            stage<T, NS>(sc, static_cast<const T*>(a.C), a.ld_c, group_offset, a.states, tile, n);
            __syncthreads();
            for (int r = 0; r < n; r += kQuad) {
                const int t = tile + r;
                const BwdRows<T, CH> now = next;
                if (t + kQuad < to) load(t + kQuad, next);
                float step[CH], in[CH], grad[CH];
#pragma unroll
                for (int i = 0; i < CH; ++i) {
                    step[i] = now.step(a, i, bias[i]);
                    in[i] = step[i] * now.x.get(i);
                    grad[i] = now.grad(a, i);
                    if (t + l.q < to) span[i] += step[i];
                }
                auto token = [&](auto j) {
                    constexpr int J = decltype(j)::value;
                    if (t + J >= to) return;
                    float bm[NS], cm[NS];
                    lds_row<NS>(sb + (r + J) * NP + l.q * NS, bm);
                    lds_row<NS>(sc + (r + J) * NP + l.q * NS, cm);
#pragma unroll
                    for (int i = 0; i < CH; ++i) {
                        const float sj = quad_get<J>(step[i]), ij = quad_get<J>(in[i]), gj = quad_get<J>(grad[i]);
#pragma unroll
                        for (int s = 0; s < NS; ++s) {
                            const float decay = __builtin_amdgcn_exp2f(sj * a2[i][s]);
                            h[i][s] = fmaf(decay, h[i][s], ij * bm[s]);
                            pass[i][s] *= decay;
                            back[i][s] = fmaf(pass[i][s], gj * cm[s], back[i][s]);
                        }
                    }
                };
                using std::integral_constant;
                token(integral_constant<int, 0>{});
                token(integral_constant<int, 1>{});
                token(integral_constant<int, 2>{});
                token(integral_constant<int, 3>{});
            }
        }
    };
    auto put = [&](float* m, const float (&v)[CH][NS]) {
#pragma unroll
        for (int i = 0; i < CH; ++i)
#pragma unroll
            for (int s = 0; s < NS; ++s)
                if (l.live[i]) m[((int64_t)chunk * a.channels + (l.c + i)) * NP + l.q * NS + s] = v[i][s];
    };
    auto put_forward = [&]() {
        put(a.carry, h);
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            span[i] = quad_sum(span[i]);
            if (l.live[i] && l.q == 0) a.span[(int64_t)chunk * a.channels + l.c + i] = span[i];
        }
    };
    if (flags & kFromBefore) {
        const int stop = min(end0, rows.hi);
        const bool ends = p.d_final && end0 <= rows.hi;
        load_state<NS, CH>(nullptr, a, l, 0, h);
        walk(rows.lo, stop);
        float d[CH][NS];      // where the sequence ends here, its final state's gradient comes back through all of its rows
        load_state<NS, CH>(ends ? p.d_final : nullptr, a, l, b0, d);
        // A growing decay's product over the rows may pass fp32's range where what it multiplies is zero or small:
        // the gradient of such a state (marked by a NaN) is taken back row by row.
        bool over = false;
#pragma unroll
        for (int i = 0; i < CH; ++i)
#pragma unroll
            for (int s = 0; s < NS; ++s) {
                if (ends) back[i][s] = fmaf(pass[i][s], d[i][s], back[i][s]);
                back[i][s] = pass[i][s] <= kLargest ? back[i][s] : __builtin_nanf("");
                over |= back[i][s] != back[i][s];
            }
        if (__any(over)) {
            const BwdPlaces<T, CH> place(a, l, 0);
            for (int t = stop - 1; t >= rows.lo; --t) {
                BwdRows<T, CH> row;
                place.load_in(a, t, row);
                place.load_grad(p, t, row);
                const T* c = static_cast<const T*>(a.C) + (int64_t)t * a.ld_c + group_offset;
#pragma unroll
                for (int i = 0; i < CH; ++i) {
                    const float step = row.step(a, i, bias[i]), grad = row.grad(a, i);
#pragma unroll
                    for (int s = 0; s < NS; ++s) {
                        const float cm = l.q * NS + s < a.states ? (float)c[l.q * NS + s] : 0.0f;
                        d[i][s] = __builtin_amdgcn_exp2f(step * a2[i][s]) * fmaf(cm, grad, d[i][s]);
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < CH; ++i)
#pragma unroll
                for (int s = 0; s < NS; ++s) back[i][s] = back[i][s] == back[i][s] ? back[i][s] : d[i][s];
        }
        put(p.back, back);
        if (flags & kThrough) put_forward();
    }
    if ((flags & kGoesOn) && !(flags & kThrough)) {
        load_state<NS, CH>(first1 >= rows.lo ? a.init : nullptr, a, l, b1, h);
        walk(max(rows.lo, first1), rows.hi);
        put_forward();
    }
}

// ---------------------------------------------------------------------------
// 2. The states behind the chunks (blockIdx.z 0) and the gradients of the
// states before them (1): one thread per channel and state.
// ---------------------------------------------------------------------------
__global__ __launch_bounds__(256) void scan_bwd_carry_kernel(ScanBwdArgs p, int padded) {
    const ScanArgs& a = p.s;
    const int64_t each = (int64_t)a.channels * padded;
    const int64_t own = (int64_t)blockIdx.x * 256 + threadIdx.x, e = min(own, each - 1);
    const int c = (int)(e / padded), n = (int)(e % padded);
    const float a2 = n < a.states ? kLog2e * a.A[(int64_t)c * a.states + n] : 0.0f;
    if (blockIdx.z == 0) carry_walk(a.carry, a, each, e, c, a2, own < each, true);
    else carry_walk(p.back, a, each, e, c, a2, own < each, false);
}

// ---------------------------------------------------------------------------
// 3. The rows' gradients
// ---------------------------------------------------------------------------

// Four values summed over the wave's lanes of the same place in their quad:
// every lane of row r of 16 holds the sum of v[kFoldOrder[r]].
__device__ __forceinline__ float fold4(float v0, float v1, float v2, float v3) {
    auto halves = [](float x, float y) {     // lanes 0-31: x over both halves; 32-63: y
        auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(y), false, false);
        return __uint_as_float(r[0]) + __uint_as_float(r[1]);
    };
    const float w0 = halves(v0, v1), w1 = halves(v2, v3);
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(w0), __float_as_uint(w1), false, false);
    float u = __uint_as_float(r[0]) + __uint_as_float(r[1]);     // rows of 16 lanes: v0, v2, v1, v3
    u += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(u), 0x124, 0xf, 0xf, true));   // rotated by 4 lanes
    u += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(u), 0x128, 0xf, 0xf, true));   // and by 8
    return u;
}
// the value that row r of 16 lanes holds: 0, 2, 1, 3
__device__ __forceinline__ int fold_place(int lane) { return (lane >> 5 & 1) | (lane >> 3 & 2); }

template <typename T, int NS, int CH, bool LOOK>
__global__ __launch_bounds__(kScanWaves * kWave, NS >= 16 ? 1 : 2) void scan_bwd_kernel(ScanBwdArgs p) {
    constexpr int NP = kQuad * NS, TB = kTileRows<NS>, GROUPS = TB / kQuad;
    extern __shared__ __align__(16) char raw_lds[];
    BwdLds<NS, CH>& lds = *reinterpret_cast<BwdLds<NS, CH>*>(raw_lds);
    const ScanArgs& a = p.s;
    const int block = blockIdx.x % a.blocks, chunk = blockIdx.x / a.blocks;
    const int wave = uniform(threadIdx.x / kWave), lane = threadIdx.x % kWave;

    if (chunk >= a.chunks) {
        // workgroups behind the chunks': the states of sequences without rows pass from one end to the other
        const int64_t each = (int64_t)a.channels * a.states;
        const int extra = (int)gridDim.x - a.blocks * a.chunks;
        for (int b = blockIdx.x - a.blocks * a.chunks; b < a.seq.count; b += extra) {
            if (a.seq.first(b + 1) > a.seq.first(b)) continue;
            for (int64_t i = threadIdx.x; i < each; i += blockDim.x)
                p.d_init[b * each + i] = p.d_final ? p.d_final[b * each + i] : 0.0f;
        }
        return;
    }

    Lane<CH> l;
    l.init(a, block, wave);
    const int group = block / a.group_blocks, group_block = block % a.group_blocks;
    const ChunkRows rows(a, chunk);
    float da[CH][NS] = {}, dd[CH] = {}, dbias[CH] = {};

    if (rows.lo < rows.hi) {
        float a2[CH][NS], bias[CH], skip[CH];
        load_decay<NS, CH>(a, l, a2);
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            bias[i] = a.dt_bias ? a.dt_bias[l.c + i] : 0.0f;
            skip[i] = a.D ? a.D[l.c + i] : 0.0f;
        }
        for (int i = threadIdx.x; i < (rows.hi - rows.lo) * NP; i += kScanWaves * kWave) {
            const int r = i / NP, s = i % NP;
            const bool in = s < a.states;
            const int64_t at = (int64_t)group * a.states + s;
            lds.b[i] = in ? (float)(static_cast<const T*>(a.B) + (int64_t)(rows.lo + r) * a.ld_b)[at] : 0.0f;
            lds.c[i] = in ? (float)(static_cast<const T*>(a.C) + (int64_t)(rows.lo + r) * a.ld_c)[at] : 0.0f;
        }
        __syncthreads();

        const BwdPlaces<T, CH> whole(a, l, l.q);
        // one row of a sequence's part of the chunk: a chunk or a sequence before it left the state
        auto start = [&](int b, bool begins, float (&h)[CH][NS]) {
            if (begins) {
                load_state<NS, CH>(a.init, a, l, b, h);
                return;
            }
            if (chunk) carried<NS, CH>(a.carry, a, l, a2, chunk - 1, -1, LOOK, h);
#pragma unroll
            for (int i = 0; i < CH; ++i)
#pragma unroll
                for (int s = 0; s < NS; ++s) h[i][s] = chunk && l.live[i] ? h[i][s] : 0.0f;
        };

        // Forwards: the state before every tile of a sequence but its first, which start() gives.  Each
        // follows TB rows of its own, so there are at most Q / TB.
        int slot = 0;
        for (int t = rows.lo; t < rows.hi;) {
            const SeqMap::Found f = a.seq.at(t);
            const int b = f.b, first = f.first, stop = min(max(f.end, t + 1), rows.hi);
            const int walk = (stop - t - 1) / TB * TB;      // rows of all tiles but the last
            if (walk) {
                float h[CH][NS];
                start(b, t == first, h);
                BwdRows<T, CH> next;
                whole.load_in(a, t, next);
                for (int r = 0; r < walk; r += kQuad) {
                    const BwdRows<T, CH> now = next;
                    if (r + kQuad < walk) whole.load_in(a, t + r + kQuad, next);
                    float step[CH], in[CH];
#pragma unroll
                    for (int i = 0; i < CH; ++i) {
                        step[i] = l.live[i] ? now.step(a, i, bias[i]) : 0.0f;
                        in[i] = l.live[i] ? step[i] * now.x.get(i) : 0.0f;
                    }
                    auto token = [&](auto j) {
                        constexpr int J = decltype(j)::value;
                        float bm[NS];
                        lds_row<NS>(lds.b + (t - rows.lo + r + J) * NP + l.q * NS, bm);
#pragma unroll
                        for (int i = 0; i < CH; ++i) {
                            const float sj = quad_get<J>(step[i]), ij = quad_get<J>(in[i]);
#pragma unroll
                            for (int s = 0; s < NS; ++s)
                                h[i][s] = fmaf(__builtin_amdgcn_exp2f(sj * a2[i][s]), h[i][s], ij * bm[s]);
                        }
                    };
                    using std::integral_constant;
                    token(integral_constant<int, 0>{});
                    token(integral_constant<int, 1>{});
                    token(integral_constant<int, 2>{});
                    token(integral_constant<int, 3>{});
                    if ((r + kQuad) % TB == 0) {
#pragma unroll
                        for (int i = 0; i < CH; ++i)
#pragma unroll
                            for (int s = 0; s < NS; ++s) lds.state[wave][slot][i * NS + s][lane] = h[i][s];
                        ++slot;
                    }
                }
            }
            t = stop;
        }

        // Backwards, sequence by sequence, tile by tile
        for (int stop = rows.hi; stop > rows.lo;) {
            const SeqMap::Found f = a.seq.at(stop - 1);
            const int b = f.b, first = f.first, end = f.end;
            const int from = max(min(first, stop - 1), rows.lo);
            float r[CH][NS];     // a g of the row behind: what the state's gradient receives from there
            if (end > stop) {
                if (chunk + 1 < a.chunks) carried<NS, CH>(p.back, a, l, a2, chunk + 1, 1, LOOK, r);
#pragma unroll
                for (int i = 0; i < CH; ++i)
#pragma unroll
                    for (int s = 0; s < NS; ++s) r[i][s] = chunk + 1 < a.chunks && l.live[i] ? r[i][s] : 0.0f;
            } else {
                load_state<NS, CH>(p.d_final, a, l, b, r);
            }
            const int tiles = (stop - from + TB - 1) / TB;
            BwdRows<T, CH> next[GROUPS];
            {
                const int t0 = from + (tiles - 1) * TB;
#pragma unroll
                for (int g = 0; g < GROUPS; ++g) {
                    const int t = t0 + g * kQuad;
                    if (t >= stop) {
                        next[g] = next[0];      // not used
                        continue;
                    }
                    const BwdPlaces<T, CH> last(a, l, min(l.q, stop - 1 - t));
                    last.load_in(a, t, next[g]);
                    last.load_grad(p, t, next[g]);
                }
            }
            for (int k = tiles - 1; k >= 0; --k) {
                const int t0 = from + k * TB, n = min(TB, stop - t0), r0 = t0 - rows.lo;
                BwdRows<T, CH> now[GROUPS];
                float step[GROUPS][CH], in[GROUPS][CH], grad[GROUPS][CH];
#pragma unroll
                for (int g = 0; g < GROUPS; ++g) {
                    now[g] = next[g];
#pragma unroll
                    for (int i = 0; i < CH; ++i) {
                        step[g][i] = now[g].dt.get(i) + bias[i];
                        grad[g][i] = now[g].dy.get(i);
                    }
                    if (a.softplus)
#pragma unroll
                        for (int i = 0; i < CH; ++i) step[g][i] = softplus(step[g][i]);
                    if (a.z)
#pragma unroll
                        for (int i = 0; i < CH; ++i) grad[g][i] *= now[g].z.get(i) * sigmoid(now[g].z.get(i));
#pragma unroll
                    for (int i = 0; i < CH; ++i) {
                        step[g][i] = l.live[i] ? step[g][i] : 0.0f;
                        in[g][i] = l.live[i] ? step[g][i] * now[g].x.get(i) : 0.0f;
                        grad[g][i] = l.live[i] ? grad[g][i] : 0.0f;
                    }
                }
                float h0[CH][NS], h[TB][CH][NS];
                if (k > 0) {
                    slot = max(slot - 1, 0);
#pragma unroll
                    for (int i = 0; i < CH; ++i)
#pragma unroll
                        for (int s = 0; s < NS; ++s) h0[i][s] = lds.state[wave][slot][i * NS + s][lane];
                } else {
                    start(b, from == first, h0);
                }

                auto forward = [&](auto j) {
                    constexpr int J = decltype(j)::value, G = J / kQuad;
                    __builtin_amdgcn_sched_barrier(0);     // rows side by side would not fit the registers
                    if (J >= n) return;
                    float bm[NS];
                    lds_row<NS>(lds.b + (r0 + J) * NP + l.q * NS, bm);
#pragma unroll
                    for (int i = 0; i < CH; ++i) {
                        const float sj = quad_get<J % kQuad>(step[G][i]), ij = quad_get<J % kQuad>(in[G][i]);
#pragma unroll
                        for (int s = 0; s < NS; ++s)
                            h[J][i][s] = fmaf(__builtin_amdgcn_exp2f(sj * a2[i][s]), J == 0 ? h0[i][s] : h[J > 0 ? J - 1 : 0][i][s], ij * bm[s]);
                    }
                };
                // a group's sums over the states, in each lane of the quad its part: of g B, q A and C h
                float du[kQuad][CH], ds[kQuad][CH], sum[kQuad][CH];
                auto clear = [&]() {
#pragma unroll
                    for (int j = 0; j < kQuad; ++j)
#pragma unroll
                        for (int i = 0; i < CH; ++i) du[j][i] = ds[j][i] = sum[j][i] = 0.0f;
                };
                auto backward = [&](auto j) {
                    constexpr int J = decltype(j)::value, G = J / kQuad;
                    __builtin_amdgcn_sched_barrier(0);
                    if (J >= n) return;
                    float bm[NS], cm[NS], v[2 * NS];
                    lds_row<NS>(lds.b + (r0 + J) * NP + l.q * NS, bm);
                    lds_row<NS>(lds.c + (r0 + J) * NP + l.q * NS, cm);
#pragma unroll
                    for (int s = 0; s < 2 * NS; ++s) v[s] = 0.0f;
#pragma unroll
                    for (int i = 0; i < CH; ++i) {
                        const float sj = quad_get<J % kQuad>(step[G][i]), ij = quad_get<J % kQuad>(in[G][i]),
                                    gj = quad_get<J % kQuad>(grad[G][i]);
                        float u = 0.0f, w = 0.0f, y = 0.0f;
#pragma unroll
                        for (int s = 0; s < NS; ++s) {
                            const float g = fmaf(cm[s], gj, r[i][s]);
                            v[s] = fmaf(g, ij, v[s]);
                            v[NS + s] = fmaf(h[J][i][s], gj, v[NS + s]);
                            u = fmaf(g, bm[s], u);
                            y = fmaf(cm[s], h[J][i][s], y);
                            r[i][s] = __builtin_amdgcn_exp2f(sj * a2[i][s]) * g;
                            const float q = r[i][s] * (J == 0 ? h0[i][s] : h[J > 0 ? J - 1 : 0][i][s]);
                            w = fmaf(q, a2[i][s], w);
                            da[i][s] = fmaf(q, sj, da[i][s]);
                        }
                        du[J % kQuad][i] = u;
                        ds[J % kQuad][i] = w;
                        sum[J % kQuad][i] = y;
                    }
#pragma unroll
                    for (int f = 0; f < 2 * NS; f += 4) {
                        const float folded = fold4(v[f], v[f + 1], v[f + 2], v[f + 3]);
                        if ((lane & 12) == 0) {
                            const int at = f + fold_place(lane);
                            lds.part[wave][J][at < NS ? l.q * NS + at : NP + l.q * NS + at - NS] = folded;
                        }
                    }
                };
                // The next tile's rows are loaded behind the stores of this tile's upper group, and arrive
                // before those of its lower one.
                auto fetch = [&]() {
                    if (k == 0) return;
#pragma unroll
                    for (int g = 0; g < GROUPS; ++g) {
                        whole.load_in(a, t0 - TB + g * kQuad, next[g]);
                        whole.load_grad(p, t0 - TB + g * kQuad, next[g]);
                    }
                };
                auto finish = [&](auto group_of_rows) {
                    constexpr int G = decltype(group_of_rows)::value;
                    const int t = t0 + G * kQuad;
                    if (G * kQuad >= n) return;
                    auto over_quad = [&](const float (&v)[kQuad][CH], int i) { return quad_sums(v[0][i], v[1][i], v[2][i], v[3][i], l.q); };
                    float dx[CH], ddt[CH], dz[CH];
                    const bool mine = G * kQuad + l.q < n;
#pragma unroll
                    for (int i = 0; i < CH; ++i) {
                        const float x = now[G].x.get(i), u = over_quad(du, i), w = over_quad(ds, i);
                        dx[i] = fmaf(u, step[G][i], skip[i] * grad[G][i]);
                        ddt[i] = fmaf(u, x, w * (1.0f / kLog2e));
                        if (a.softplus) ddt[i] *= sigmoid(now[G].dt.get(i) + bias[i]);
                        if (a.z) {
                            const float z = now[G].z.get(i), sig = sigmoid(z);
                            dz[i] = now[G].dy.get(i) * fmaf(skip[i], x, over_quad(sum, i)) * sig * fmaf(z, 1.0f - sig, 1.0f);
                        }
                        if (mine) {
                            dd[i] = fmaf(grad[G][i], x, dd[i]);
                            dbias[i] += ddt[i];
                        }
                    }
                    if constexpr (G == 0)
#pragma unroll
                        for (int g = 0; g < GROUPS; ++g) next[g].wait();
                    if (mine) {
                        store_channels<T, CH>(whole.dense.at(p.dx, a.channels, t), l.live, dx);
                        store_channels<T, CH>(whole.dense.at(p.ddt, a.channels, t), l.live, ddt);
                        if (a.z) store_channels<T, CH>(whole.dense.at(p.dz, a.channels, t), l.live, dz);
                    }
                };
                using std::integral_constant;
                forward(integral_constant<int, 0>{});
                forward(integral_constant<int, 1>{});
                forward(integral_constant<int, 2>{});
                forward(integral_constant<int, 3>{});
                if constexpr (TB == 8) {
                    forward(integral_constant<int, 4>{});
                    forward(integral_constant<int, 5>{});
                    forward(integral_constant<int, 6>{});
                    forward(integral_constant<int, 7>{});
                    clear();
                    backward(integral_constant<int, 7>{});
                    backward(integral_constant<int, 6>{});
                    backward(integral_constant<int, 5>{});
                    backward(integral_constant<int, 4>{});
                    finish(integral_constant<int, 1>{});
                }
                clear();
                fetch();
                backward(integral_constant<int, 3>{});
                backward(integral_constant<int, 2>{});
                backward(integral_constant<int, 1>{});
                backward(integral_constant<int, 0>{});
                finish(integral_constant<int, 0>{});

                // the waves' sums of dB and dC
                __syncthreads();
                for (int i = threadIdx.x; i < n * 2 * NP; i += kScanWaves * kWave) {
                    const int j = i / (2 * NP), m = i % (2 * NP);
                    float v = lds.part[0][j][m];
#pragma unroll
                    for (int w = 1; w < kScanWaves; ++w) v += lds.part[w][j][m];
                    p.dbc[(((int64_t)group_block * a.seq.tokens + t0 + j) * p.groups + group) * (2 * NP) + m] = v;
                }
                __syncthreads();
            }
            if (p.d_init && from == first) {
#pragma unroll
                for (int i = 0; i < CH; ++i)
#pragma unroll
                    for (int s = 0; s < NS; ++s) {
                        const int m = l.q * NS + s;
                        if (l.live[i] && m < a.states) p.d_init[((int64_t)b * a.channels + (l.c + i)) * a.states + m] = r[i][s];
                    }
            }
            stop = from;
        }
    }

#pragma unroll
    for (int i = 0; i < CH; ++i) {
        dd[i] = quad_sum(dd[i]);
        dbias[i] = quad_sum(dbias[i]);
        if (!l.live[i]) continue;
        const int64_t at = (int64_t)chunk * a.channels + (l.c + i);
#pragma unroll
        for (int s = 0; s < NS; ++s) p.da_part[at * NP + l.q * NS + s] = da[i][s];
        if (l.q == 0) {
            p.dd_part[2 * at] = dd[i];
            p.dd_part[2 * at + 1] = dbias[i];
        }
    }
}

// ---------------------------------------------------------------------------
// 4. Sums.  Workgroups 0 to param_blocks - 1: 64 channels' states (or
// channels) each, a wave for every fourth chunk; the others dB and dC.
// ---------------------------------------------------------------------------
template <typename T>
__global__ __launch_bounds__(kScanWaves * kWave) void scan_bwd_sum_kernel(ScanBwdArgs p, int padded, int state_blocks, int param_blocks) {
    const ScanArgs& a = p.s;
    __shared__ float part[kScanWaves][kWave];
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    if ((int)blockIdx.x < param_blocks) {
        const bool states = (int)blockIdx.x < state_blocks;
        const int64_t each = (int64_t)a.channels * (states ? padded : 2);
        const float* m = states ? p.da_part : p.dd_part;
        const int64_t e = ((int64_t)blockIdx.x - (states ? 0 : state_blocks)) * kWave + lane;
        float v = 0.0f;
        if (e < each)
            for (int k = wave; k < a.chunks; k += kScanWaves) v += m[k * each + e];
        part[wave][lane] = v;
        __syncthreads();
        if (wave != 0 || e >= each) return;
#pragma unroll
        for (int w = 1; w < kScanWaves; ++w) v += part[w][lane];
        if (states) {
            const int64_t c = e / padded, n = e % padded;
            if (n < a.states) p.dA[c * a.states + n] = v;
        } else {
            float* out = e % 2 ? p.ddt_bias : p.dD;
            if (out) out[e / 2] = v;
        }
        return;
    }
    // dB and dC of the rows that sequences hold
    const int64_t per_row = (int64_t)p.groups * a.states;
    const int64_t lo = (int64_t)a.seq.first(0) * per_row, hi = (int64_t)a.seq.first(a.seq.count) * per_row;
    const int64_t e = ((int64_t)blockIdx.x - param_blocks) * blockDim.x + threadIdx.x;
    if (e < lo || e >= hi) return;
    const int64_t rg = e / a.states, n = e % a.states;      // row and group
    const float* m = p.dbc + rg * (2 * padded) + n;
    const int64_t next = (int64_t)a.seq.tokens * p.groups * (2 * padded);
    float b = 0.0f, c = 0.0f;
    for (int k = 0; k < a.group_blocks; ++k, m += next) {
        b += m[0];
        c += m[padded];
    }
    static_cast<T*>(p.dB)[e] = (T)b;
    static_cast<T*>(p.dC)[e] = (T)c;
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
struct BwdPlan {
    int64_t chunk = 0, chunks = 0, blocks = 0, group_blocks = 0;
    int ns = 0, ch = 0;
    size_t carry = 0, span = 0, flags = 0, dbc = 0, da = 0, dd = 0, bytes = 0;
};

size_t round16(size_t n) { return (n + 15) / 16 * 16; }

BwdPlan plan_bwd(const im2win_scan_desc* d) {
    BwdPlan p;
    int64_t tile = 8;
    with_states(d->states, narrow(d), [&](auto ns, auto ch) {
        p.ns = decltype(ns)::value;
        p.ch = decltype(ch)::value;
        p.chunk = kChunkRows<decltype(ns)::value>;
        tile = kTileRows<decltype(ns)::value>;
    });
    const int64_t per_block = kScanWaves * (kWave / kQuad) * p.ch;
    p.group_blocks = (d->channels / d->groups + per_block - 1) / per_block;
    p.blocks = d->groups * p.group_blocks;
    if (d->tokens == 0) return p;
    // the longest chunk the LDS holds, halved while that leaves fewer than two workgroups for each CU
    while (p.chunk > 2 * tile && p.blocks * ((d->tokens + p.chunk - 1) / p.chunk) < 512)
        p.chunk = std::max(p.chunk / 2 / tile, int64_t(2)) * tile;
    p.chunk = std::min(p.chunk, d->tokens);
    p.chunks = (d->tokens + p.chunk - 1) / p.chunk;
    const int64_t np = kQuad * p.ns;
    p.carry = round16((size_t)(p.chunks * d->channels * np) * 4);
    p.span = round16((size_t)(p.chunks * d->channels) * 4);
    p.flags = round16((size_t)p.chunks * 4);
    p.dbc = round16((size_t)(p.group_blocks * d->tokens * d->groups * 2 * np) * 4);
    p.da = p.carry;
    p.dd = 2 * p.span;
    p.bytes = 2 * p.carry + p.span + p.flags + p.dbc + p.da + p.dd;
    return p;
}

// States of a lane up to which chunks may look for themselves instead of a
// carry kernel, in three walks each: 16 chunks a sequence 130 us with the kernel
// and 126 without, 32 chunks 214 and 229; of 64 states, 63 chunks in 9 ragged
// sequences 104 and 134.  One ragged sequence that holds nearly all of 63 chunks
// costs more (4000 x 2048 x 16: 213 us with the kernel, 258 without; 1000 x 420 x
// 32: 68 and 111), many gain (2003 x 2048 x 16 in 17 sequences: 140 and 133).
constexpr int kLookStates = 8;

constexpr int kEmptyBlocks = 32;

template <typename F>
void with_type(int32_t dtype, F f) {
    if (dtype == IM2WIN_F32) f(float{});
    else f(bf16{});
}

}  // namespace
}  // namespace im2win

using namespace im2win;

extern "C" {

int im2win_selective_scan_backward_workspace_bytes(const im2win_scan_desc* d, size_t* bytes) {
    int rc = check_scan(d, true, nullptr, false);
    if (rc) return rc;
    if (!bytes) return fail(IM2WIN_ENULL, "bytes is NULL");
    *bytes = plan_bwd(d).bytes;
    return ok();
}

int im2win_selective_scan_backward(const im2win_scan_desc* d, const void* dy, const void* x, const void* dt,
                                   const float* A, const void* B, const void* C, const float* D, const void* z,
                                   const float* dt_bias, const int32_t* seq_starts, const float* initial_state,
                                   const float* d_final_state, void* dx, void* ddt, float* dA, void* dB, void* dC,
                                   float* dD, void* dz, float* ddt_bias, float* d_initial_state, void* workspace,
                                   size_t workspace_bytes, void* stream) {
    int rc = check_scan(d, true, seq_starts, true);
    if (rc || (rc = check_scan_inputs(d, x, dt, A, B, C, D, z, dt_bias))) return rc;
    const size_t e = d->dtype == IM2WIN_F32 ? 4 : 2;
    if (d->tokens && ((rc = need_ptr(dy, e, "dy")) || (rc = need_ptr(dx, e, "dx")) || (rc = need_ptr(ddt, e, "ddt")) ||
                      (rc = need_ptr(dB, e, "dB")) || (rc = need_ptr(dC, e, "dC")) ||
                      (z && (rc = need_ptr(dz, e, "dz")))))
        return rc;
    if ((rc = need_ptr(dA, 4, "dA")) || (rc = may_ptr(dD, 4, "dD")) || (rc = may_ptr(ddt_bias, 4, "ddt_bias")) ||
        (rc = may_ptr(initial_state, 4, "initial_state")) || (rc = may_ptr(d_final_state, 4, "d_final_state")) ||
        (rc = may_ptr(d_initial_state, 4, "d_initial_state")))
        return rc;
    const BwdPlan p = plan_bwd(d);
    if (p.bytes && (rc = need_ptr(workspace, 16, "workspace"))) return rc;
    if (workspace_bytes < p.bytes)
        return fail(IM2WIN_EWORKSPACE, "workspace holds %zu bytes, the gradients need %zu", workspace_bytes, p.bytes);
    ScanBwdArgs b{};
    b.s = scan_args(d, x, dt, A, B, C, D, z, dt_bias, p.ch);
    b.s.init = initial_state;
    b.s.seq = make_seq_map(d->tokens, d->sequences, seq_starts);
    b.s.chunk = (int)p.chunk; b.s.chunks = (int)p.chunks;
    b.dy = dy; b.d_final = d_final_state; b.dx = dx; b.ddt = ddt; b.dA = dA; b.dB = dB; b.dC = dC; b.dD = dD;
    b.dz = dz; b.ddt_bias = ddt_bias; b.d_init = d_initial_state;
    b.groups = (int)d->groups;
    char* ws = static_cast<char*>(workspace);
    auto take = [&](size_t n) { char* q = ws; ws += n; return q; };
    if (p.bytes) {
        b.s.carry = reinterpret_cast<float*>(take(p.carry));
        b.back = reinterpret_cast<float*>(take(p.carry));
        b.s.span = reinterpret_cast<float*>(take(p.span));
        b.s.flags = reinterpret_cast<int*>(take(p.flags));
        b.dbc = reinterpret_cast<float*>(take(p.dbc));
        b.da_part = reinterpret_cast<float*>(take(p.da));
        b.dd_part = reinterpret_cast<float*>(take(p.dd));
    }
    const int64_t grid = p.blocks * p.chunks;
    const int64_t extra = d_initial_state && (seq_starts || d->tokens == 0) ? std::min<int64_t>(d->sequences, kEmptyBlocks) : 0;
    const int64_t np = kQuad * p.ns;
    const int64_t state_blocks = (d->channels * np + kWave - 1) / kWave;
    const int64_t param_blocks = state_blocks + (2 * d->channels + kWave - 1) / kWave;
    const int64_t sums = param_blocks + (d->tokens * d->groups * d->states + kScanWaves * kWave - 1) / (kScanWaves * kWave);
    if ((rc = check_launch(std::max(grid + extra, sums), kScanWaves * kWave, "selective_scan_backward"))) return rc;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const bool look = p.ns <= kLookStates && look_back(p.chunks, d->sequences, seq_starts != nullptr, 16);
    int hip = 0;
    with_type(d->dtype, [&](auto t) {
        using T = decltype(t);
        with_states(d->states, narrow(d), [&](auto ns, auto ch) {
            constexpr int NS = decltype(ns)::value, CH = decltype(ch)::value;
            const dim3 threads(kScanWaves * kWave);
            if (p.chunks > 1) {
                hipLaunchKernelGGL((scan_bwd_summary_kernel<T, NS, CH>), dim3((unsigned)grid), threads, 0, s, b);
                if (!look)
                    hipLaunchKernelGGL(scan_bwd_carry_kernel, dim3((unsigned)((d->channels * np + 255) / 256), carry_pieces(p.chunks), 2), dim3(256), 0, s,
                                       b, (int)np);
            }
            if (grid + extra) {
                constexpr int bytes = (int)sizeof(BwdLds<NS, CH>);
                static_assert(bytes <= 160 * 1024, "LDS of a CU");
                auto launch = [&](auto kernel) {
                    if (bytes > 64 * 1024)
                        hip = (int)hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
                    if (!hip) hipLaunchKernelGGL(kernel, dim3((unsigned)(grid + extra)), threads, bytes, s, b);
                };
                if constexpr (NS <= kLookStates) {
                    if (look) launch(&scan_bwd_kernel<T, NS, CH, true>);
                    else launch(&scan_bwd_kernel<T, NS, CH, false>);
                } else {
                    launch(&scan_bwd_kernel<T, NS, CH, false>);
                }
            }
        });
        if (!hip)
            hipLaunchKernelGGL((scan_bwd_sum_kernel<T>), dim3((unsigned)sums), dim3(kScanWaves * kWave), 0, s, b, (int)np,
                               (int)state_blocks, (int)param_blocks);
    });
    if (hip) return fail(IM2WIN_EHIP, "LDS size: %s", hipGetErrorString((hipError_t)hip));
    return launched("selective_scan_backward");
}

}  // extern "C"
