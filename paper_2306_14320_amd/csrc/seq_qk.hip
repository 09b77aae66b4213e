// Root-mean-square norm of the queries and keys of each head and the rotation
// by their positions, in one pass, and its gradients.  For every head's
// channels x of a row t,
//   r = rsqrt(mean(x^2) + eps),  u = x r w,
//   (y_p, y_p') = (u_p cos - u_p' sin, u_p' cos + u_p sin)
// for the pairs (p, p') of the first rot_dim channels, of the angle
// positions[t] freqs[p]; the channels behind them are not rotated.  Gradients,
// with du the rotation of dy by the opposite angle, n = x r and g = du w:
//   dx = r (g - n mean(g n)),  dw = sum over rows and heads of du n.
//
// Bound by memory (16384 rows of 20 heads of 128 bf16: 35.8 us a call, 4.7 TB/s, where
// a copy has 5.1) with vector units busy for 88% (the gradients, 4001 rows of 15 heads
// of 80 fp32: 16.1 us, 3.6 TB/s, and 5.4 for the weights' sums): a head's channels are
// read once, into the registers of a few neighbouring lanes, as pairs: a lane holds V pairs, 16 bytes of the
// first channels and 16 of their partners, so that the rotation needs no
// exchange and the sum of squares a few within the group.  The wave's lanes
// take one angle each and share them through LDS; all heads of the row use them.
//
// The angle of a far position has more digits than fp32: the turns are taken
// in fp64, and what is left behind the whole ones (at most half a turn) in
// two parts of fp32, the second of which turns the first's cosine and sine on.
#include "seq_common.h"

#include <algorithm>
#include <type_traits>

namespace im2win {
namespace {

constexpr int kMaxPairs = 256;     // head sizes up to 512
constexpr int kWavesPer = 4;       // waves of a workgroup

struct QkArgs {
    const void *q, *k;             // forward: inputs; backward: the same
    const void *dq, *dk;           // gradients of the outputs
    const float *wq, *wk;
    const int32_t* pos;
    const float* freqs;
    void *yq, *yk;                 // outputs, or gradients of the inputs
    float* part;                   // workgroup x (wq, wk): sums of the weights' gradients
    int64_t ld_q, ld_k;
    int tokens, q_heads, k_heads, dim, rot;
    int lanes;                     // of a head, a power of two
    int parts;                     // waves that share a row's heads
    float eps, inv_d;
};

// V elements in flight: 16 or 8 bytes at any alignment, or one element
template <typename T, int V>
struct Run {
    uint32_t u[V * sizeof(T) < 4 ? 1 : V * sizeof(T) / 4];
    __device__ __forceinline__ void load(const T* p) {
        if constexpr (V * sizeof(T) < 4) u[0] = __builtin_bit_cast(uint16_t, *p);
        else __builtin_memcpy(u, p, V * sizeof(T));
    }
    __device__ __forceinline__ float get(int i) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(u[i]);
        else return __uint_as_float(i % 2 ? u[i / 2] & 0xffff0000u : u[i / 2] << 16);
    }
};
template <int V>
__device__ __forceinline__ void put(float* p, const float (&v)[V]) { __builtin_memcpy(p, v, 4 * V); }
template <int V>
__device__ __forceinline__ void put(bf16* p, const float (&v)[V]) {
    if constexpr (V == 1) {
        *p = (bf16)v[0];
    } else {
        uint32_t u[V / 2];
#pragma unroll
        for (int i = 0; i < V / 2; ++i) u[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
        __builtin_memcpy(p, u, 2 * V);
    }
}

// V pairs of a head's channels: neighbours (2p, 2p + 1), or p and its partner
// half of the rotated (or of the other) channels on
template <typename T, int V, bool NEAR>
struct Pairs {
    Run<T, V> a, b;
    __device__ __forceinline__ void load(const T* p, int lo, int hi) {
        if constexpr (NEAR && V > 1) {
            a.load(p + lo);
            b.load(p + lo + V);
        } else {
            a.load(p + lo);
            b.load(p + hi);
        }
    }
    __device__ __forceinline__ void get(float (&x)[V], float (&y)[V]) const {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if constexpr (NEAR && V > 1) {
                x[i] = 2 * i < V ? a.get(2 * i) : b.get(2 * i - V);
                y[i] = 2 * i < V ? a.get(2 * i + 1) : b.get(2 * i + 1 - V);
            } else {
                x[i] = a.get(i);
                y[i] = b.get(i);
            }
        }
    }
};
template <int V, bool NEAR, typename T>
__device__ __forceinline__ void put_pairs(T* p, int lo, int hi, const float (&x)[V], const float (&y)[V]) {
    if constexpr (NEAR && V > 1) {
        float f[V], s[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            f[i] = i % 2 ? y[i / 2] : x[i / 2];
            s[i] = i % 2 ? y[(V + i) / 2] : x[(V + i) / 2];
        }
        put(p + lo, f);
        put(p + lo + V, s);
    } else {
        put(p + lo, x);
        put(p + hi, y);
    }
}

// One of two registers (written as a conditional of two array elements, the
// compiler selects between addresses and puts the arrays into scratch)
__device__ __forceinline__ float pick(bool first, float a, float b) { return first ? a : b; }

// The sum over the lanes of a head
__device__ __forceinline__ float head_sum(float v, int lanes) {
    for (int m = 1; m < lanes; m *= 2) v += __shfl_xor(v, m);
    return v;
}

// A lane's place: J units of V pairs, from the pair lane + G j on
template <int V, int J, bool NEAR>
struct Place {
    int lo[J], hi[J], pair[J];
    bool on[J];
    __device__ __forceinline__ Place(int lane, int lanes, int dim, int rot) {
#pragma unroll
        for (int j = 0; j < J; ++j) {
            pair[j] = (lane % lanes + j * lanes) * V;
            on[j] = pair[j] < dim / 2;
            const int p = on[j] ? pair[j] : 0;
            if constexpr (NEAR) {
                lo[j] = 2 * p;
                hi[j] = 2 * p + 1;
            } else {
                lo[j] = p < rot / 2 ? p : rot / 2 + p;
                hi[j] = p < rot / 2 ? rot / 2 + p : dim / 2 + p;
            }
            pair[j] = p;
        }
    }
};

// The wave's LDS accesses before and behind are in that order (its own part, so no barrier).
__device__ __forceinline__ void wave_order() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// cos and sin of the row's angles, one a lane, into the wave's part of LDS
__device__ __forceinline__ void angles(const QkArgs& a, int t, float* cs, float* sn) {
    const int lane = threadIdx.x % kWave;
    const double at = a.rot ? (double)a.pos[t] : 0.0;
    for (int p = lane; p < a.rot / 2; p += kWave) {
        double turns = at * ((double)a.freqs[p] * 0.15915494309189533577);
        turns -= __builtin_rint(turns);
        const float near = (float)turns, rest = (float)(turns - (double)near) * 6.28318530717958648f;
        float s, c;
        sincospif(2.0f * near, &s, &c);
        cs[p] = fmaf(-s, rest, c);
        sn[p] = fmaf(c, rest, s);
    }
}

template <int V, int J>
__device__ __forceinline__ void take_angles(const float* cs, const float* sn, const int (&pair)[J], int rot, float (&c)[J][V], float (&s)[J][V]) {
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const bool in = pair[j] + i < rot / 2;
            c[j][i] = in ? cs[pair[j] + i] : 1.0f;
            s[j][i] = in ? sn[pair[j] + i] : 0.0f;
        }
}

template <typename T, int V, int J, bool NEAR>
__global__ __launch_bounds__(kWavesPer * kWave) void qk_norm_rope_kernel(QkArgs a) {
    __shared__ float cs[kWavesPer][kMaxPairs], sn[kWavesPer][kMaxPairs];
    const int wave = uniform(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    const int64_t w = (int64_t)blockIdx.x * kWavesPer + wave;
    const int t = uniform((int)(w / a.parts)), part = uniform((int)(w % a.parts));
    if (t >= a.tokens) return;
    const Place<V, J, NEAR> at(lane, a.lanes, a.dim, a.rot);
    const int heads = a.q_heads + a.k_heads, per = kWave / a.lanes;
    const T* q = static_cast<const T*>(a.q) + t * a.ld_q;
    const T* k = static_cast<const T*>(a.k) + t * a.ld_k;
    T* yq = static_cast<T*>(a.yq) + (int64_t)t * a.q_heads * a.dim;
    T* yk = static_cast<T*>(a.yk) + (int64_t)t * a.k_heads * a.dim;
    auto source = [&](int h) { return h < a.q_heads ? q + (int64_t)h * a.dim : k + (int64_t)(h - a.q_heads) * a.dim; };

    int h = part * per + lane / a.lanes;
    Pairs<T, V, NEAR> x[J], next[J];
    auto fetch = [&](int head, Pairs<T, V, NEAR> (&o)[J]) {
        const T* p = source(head < heads ? head : heads - 1);
#pragma unroll
        for (int j = 0; j < J; ++j) o[j].load(p, at.lo[j], at.hi[j]);
    };
    fetch(h, x);
    float wq[J][2][V], wk[J][2][V];
#pragma unroll
    for (int j = 0; j < J; ++j) {
        Pairs<float, V, NEAR> f;
        f.load(a.wq, at.lo[j], at.hi[j]);
        f.get(wq[j][0], wq[j][1]);
        f.load(a.wk, at.lo[j], at.hi[j]);
        f.get(wk[j][0], wk[j][1]);
    }
    angles(a, t, cs[wave], sn[wave]);
    wave_order();
    float c[J][V], s[J][V];
    take_angles<V, J>(cs[wave], sn[wave], at.pair, a.rot, c, s);

    for (int first = part * per; first < heads; first += a.parts * per) {
        const int ahead = h + a.parts * per;
        if (first + a.parts * per < heads) fetch(ahead, next);
        float sum = 0.0f, lo[J][V], hi[J][V];
#pragma unroll
        for (int j = 0; j < J; ++j) {
            x[j].get(lo[j], hi[j]);
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (at.on[j]) sum = fmaf(lo[j][i], lo[j][i], fmaf(hi[j][i], hi[j][i], sum));
        }
        const float r = 1.0f / __builtin_sqrtf(fmaf(head_sum(sum, a.lanes), a.inv_d, a.eps));
        const bool isq = h < a.q_heads;
        if (h < heads) {
            T* y = isq ? yq + (int64_t)h * a.dim : yk + (int64_t)(h - a.q_heads) * a.dim;
#pragma unroll
            for (int j = 0; j < J; ++j) {
                if (!at.on[j]) continue;
                float u[V], v[V];
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float m = lo[j][i] * r * pick(isq, wq[j][0][i], wk[j][0][i]);
                    const float n = hi[j][i] * r * pick(isq, wq[j][1][i], wk[j][1][i]);
                    u[i] = fmaf(m, c[j][i], -n * s[j][i]);
                    v[i] = fmaf(n, c[j][i], m * s[j][i]);
                }
                put_pairs<V, NEAR>(y, at.lo[j], at.hi[j], u, v);
            }
        }
#pragma unroll
        for (int j = 0; j < J; ++j) x[j] = next[j];
        h = ahead;
    }
}

// Gradients: the workgroups' waves walk the rows; the weights' gradients stay
// in registers until the walk ends and are then added over lanes, waves and,
// by a second kernel, workgroups, always in the same order.
template <typename T, int V, int J, bool NEAR>
__global__ __launch_bounds__(kWavesPer * kWave) void qk_norm_rope_bwd_kernel(QkArgs a) {
    __shared__ float cs[kWavesPer][kMaxPairs], sn[kWavesPer][kMaxPairs];
    __shared__ float sums[kWavesPer][4][kMaxPairs];
    const int wave = uniform(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    const Place<V, J, NEAR> at(lane, a.lanes, a.dim, a.rot);
    const int heads = a.q_heads + a.k_heads, per = kWave / a.lanes;
    float wq[J][2][V], wk[J][2][V], gq[J][2][V], gk[J][2][V];
#pragma unroll
    for (int j = 0; j < J; ++j) {
        Pairs<float, V, NEAR> f;
        f.load(a.wq, at.lo[j], at.hi[j]);
        f.get(wq[j][0], wq[j][1]);
        f.load(a.wk, at.lo[j], at.hi[j]);
        f.get(wk[j][0], wk[j][1]);
#pragma unroll
        for (int i = 0; i < V; ++i) gq[j][0][i] = gq[j][1][i] = gk[j][0][i] = gk[j][1][i] = 0.0f;
    }
    const int64_t waves = (int64_t)gridDim.x * kWavesPer;
    for (int64_t w = (int64_t)blockIdx.x * kWavesPer + wave; w < (int64_t)a.tokens * a.parts; w += waves) {
        const int t = uniform((int)(w / a.parts)), part = uniform((int)(w % a.parts));
        const T* q = static_cast<const T*>(a.q) + t * a.ld_q;
        const T* k = static_cast<const T*>(a.k) + t * a.ld_k;
        const int64_t rq = (int64_t)t * a.q_heads * a.dim, rk = (int64_t)t * a.k_heads * a.dim;
        wave_order();
        angles(a, t, cs[wave], sn[wave]);
        wave_order();
        float c[J][V], s[J][V];
        take_angles<V, J>(cs[wave], sn[wave], at.pair, a.rot, c, s);
        for (int first = part * per; first < heads; first += a.parts * per) {
            const int h = first + lane / a.lanes, hh = h < heads ? h : heads - 1;
            const bool isq = hh < a.q_heads;
            const T* xp = isq ? q + (int64_t)hh * a.dim : k + (int64_t)(hh - a.q_heads) * a.dim;
            const int64_t off = isq ? rq + (int64_t)hh * a.dim : rk + (int64_t)(hh - a.q_heads) * a.dim;
            const T* dp = static_cast<const T*>(isq ? a.dq : a.dk) + off;
            Pairs<T, V, NEAR> x[J], d[J];
#pragma unroll
            for (int j = 0; j < J; ++j) {
                x[j].load(xp, at.lo[j], at.hi[j]);
                d[j].load(dp, at.lo[j], at.hi[j]);
            }
            float sq = 0.0f, dot = 0.0f, lo[J][V], hi[J][V], dlo[J][V], dhi[J][V];
#pragma unroll
            for (int j = 0; j < J; ++j) {
                x[j].get(lo[j], hi[j]);
                float u[V], v[V];
                d[j].get(u, v);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    dlo[j][i] = fmaf(u[i], c[j][i], v[i] * s[j][i]);
                    dhi[j][i] = fmaf(v[i], c[j][i], -u[i] * s[j][i]);
                    if (at.on[j]) {
                        sq = fmaf(lo[j][i], lo[j][i], fmaf(hi[j][i], hi[j][i], sq));
                        dot = fmaf(dlo[j][i] * pick(isq, wq[j][0][i], wk[j][0][i]), lo[j][i], fmaf(dhi[j][i] * pick(isq, wq[j][1][i], wk[j][1][i]), hi[j][i], dot));
                    }
                }
            }
            const float r = 1.0f / __builtin_sqrtf(fmaf(head_sum(sq, a.lanes), a.inv_d, a.eps));
            const float m = head_sum(dot, a.lanes) * a.inv_d * r * r;      // mean(g n) / |x's part|: dx = r (g - x m)
            if (h < heads) {
                T* y = static_cast<T*>(isq ? a.yq : a.yk) + off;
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    if (!at.on[j]) continue;
                    float u[V], v[V];
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        u[i] = r * fmaf(-lo[j][i], m, dlo[j][i] * pick(isq, wq[j][0][i], wk[j][0][i]));
                        v[i] = r * fmaf(-hi[j][i], m, dhi[j][i] * pick(isq, wq[j][1][i], wk[j][1][i]));
                        const float f = dlo[j][i] * (lo[j][i] * r), g = dhi[j][i] * (hi[j][i] * r);
                        if (isq) gq[j][0][i] += f, gq[j][1][i] += g;
                        else gk[j][0][i] += f, gk[j][1][i] += g;
                    }
                    put_pairs<V, NEAR>(y, at.lo[j], at.hi[j], u, v);
                }
            }
        }
    }
    // over the wave's heads, then the workgroup's waves
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            float v[4] = {gq[j][0][i], gq[j][1][i], gk[j][0][i], gk[j][1][i]};
            for (int m = a.lanes; m < kWave; m *= 2) {
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] += __shfl_xor(v[e], m);
            }
            if (at.on[j] && lane < a.lanes) {
#pragma unroll
                for (int e = 0; e < 4; ++e) sums[wave][e][at.pair[j] + i] = v[e];
            }
        }
    __syncthreads();
    float* out = a.part + (int64_t)blockIdx.x * 2 * a.dim;
    for (int i = threadIdx.x; i < 4 * (a.dim / 2); i += kWavesPer * kWave) {
        const int e = i / (a.dim / 2), p = i % (a.dim / 2);
        float v = 0.0f;
        for (int w = 0; w < kWavesPer; ++w) v += sums[w][e][p];
        const int lo = NEAR ? 2 * p : p < a.rot / 2 ? p : a.rot / 2 + p;
        const int hi = NEAR ? 2 * p + 1 : p < a.rot / 2 ? a.rot / 2 + p : a.dim / 2 + p;
        out[(e / 2) * a.dim + (e % 2 ? hi : lo)] = v;
    }
}

constexpr int kSumWaves = 16, kSums = 8;

// The sum of values by pairs, whose error grows with the logarithm of their number
template <int N>
__device__ __forceinline__ float added(const float (&v)[N]) {
    float s[N];
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] = v[i];
#pragma unroll
    for (int n = N / 2; n; n /= 2)
#pragma unroll
        for (int i = 0; i < n; ++i) s[i] += s[i + n];
    return s[0];
}

// dwq and dwk from the workgroups' sums
__global__ __launch_bounds__(kSumWaves * kWave) void qk_norm_rope_bwd_sum_kernel(const float* part, float* dwq, float* dwk, int blocks, int dim) {
    __shared__ float sum[kSumWaves][kWave];
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    const int c = (int)blockIdx.x * kWave + lane;
    float s[kSums] = {};
    if (c < 2 * dim) {
        for (int i = wave; i < blocks; i += kSums * kSumWaves)
#pragma unroll
            for (int j = 0; j < kSums; ++j) s[j] += i + j * kSumWaves < blocks ? part[(int64_t)(i + j * kSumWaves) * 2 * dim + c] : 0.0f;
    }
    sum[wave][lane] = added(s);
    __syncthreads();
    if (wave == 0 && c < 2 * dim) {
        float w[kSumWaves];
#pragma unroll
        for (int i = 0; i < kSumWaves; ++i) w[i] = sum[i][lane];
        (c < dim ? dwq + c : dwk + (c - dim))[0] = added(w);
    }
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
int check_desc(const im2win_qk_desc* d) {
    if (!d) return fail(IM2WIN_ENULL, "descriptor is NULL");
    if (d->q_heads < 0 || d->k_heads < 0 || d->q_heads + d->k_heads < 1 || d->q_heads > 65536 || d->k_heads > 65536)
        return fail(IM2WIN_EINVAL, "q_heads and k_heads must be 0 to 65536, one of them at least 1 (got %lld, %lld)", (long long)d->q_heads, (long long)d->k_heads);
    if (d->head_dim < 2 || d->head_dim > 2 * kMaxPairs || d->head_dim % 2)
        return fail(IM2WIN_EINVAL, "head_dim must be even, 2 to %d (got %lld)", 2 * kMaxPairs, (long long)d->head_dim);
    if (d->rot_dim < 0 || d->rot_dim > d->head_dim || d->rot_dim % 2)
        return fail(IM2WIN_EINVAL, "rot_dim must be even, 0 to head_dim (got %lld of %lld)", (long long)d->rot_dim, (long long)d->head_dim);
    int rc = check_rows(d->tokens, 1, d->dtype);
    if (rc) return rc;
    if (!(d->eps >= 0.0f)) return fail(IM2WIN_EINVAL, "eps must be >= 0 (got %g)", (double)d->eps);
    if (d->q_heads && (rc = check_ld(d->ld_q, d->q_heads * d->head_dim, "ld_q"))) return rc;
    if (d->k_heads && (rc = check_ld(d->ld_k, d->k_heads * d->head_dim, "ld_k"))) return rc;
    return IM2WIN_OK;
}

struct Shape {
    int v, j, lanes;
    int64_t parts, blocks;
};

// The widest runs of pairs that neither the middle nor the end of the rotated
// channels cuts: 16 bytes, 8, or single pairs, of which a lane takes up to four.
Shape shape_of(const im2win_qk_desc* d) {
    Shape s{};
    const int dim = (int)d->head_dim, rot = (int)d->rot_dim;
    const int most = d->dtype == IM2WIN_F32 ? 4 : 8;
    auto fits = [&](int v) { return d->interleaved ? dim / 2 % v == 0 : rot / 2 % v == 0 && (dim - rot) / 2 % v == 0; };
    s.v = fits(most) ? most : fits(4) ? 4 : 1;
    const int units = dim / 2 / s.v;
    s.lanes = 1;
    while (s.lanes < units && s.lanes < kWave) s.lanes *= 2;
    s.j = (units + s.lanes - 1) / s.lanes;
    // a wave takes a row's heads one round after the other; where rows are
    // few, several waves share them, so that the chip has some 4096
    const int64_t per = kWave / s.lanes, rounds = (d->q_heads + d->k_heads + per - 1) / per;
    s.parts = std::max<int64_t>(1, std::min(rounds, d->tokens ? 4096 / d->tokens : 1));
    s.blocks = (d->tokens * s.parts + kWavesPer - 1) / kWavesPer;
    return s;
}

// Workgroups of the gradients, whose waves walk the rows: as many as run at once,
// by the registers of the variant, so that none waits for the others (bf16 rows of
// 16384: 20 x 128, three a CU, 58 us with 768, 74 with 1024; 6 x 510 of single
// pairs in fours 100 with 768, 126 with 1024; 20 x 80 in runs of four 51 with 1280,
// 56 with 1024; 20 x 70 of single pairs 128 with 1536, 158 with 1024).  In fp32
// four a CU take runs of four (20 x 128 106 with 1024, 118 with 1280).
int64_t bwd_blocks(const Shape& s, int32_t dtype) {
    const int64_t per_cu = s.v == 8 || s.j > 1 ? 3 : s.v == 1 ? 6 : dtype == IM2WIN_F32 ? 4 : 5;
    return std::min<int64_t>(s.blocks, 256 * per_cu);
}

template <typename F>
void with_shape(const im2win_qk_desc* d, const Shape& s, F f) {
    using std::integral_constant;
    auto near = [&](auto t, auto v, auto j) {
        if (d->interleaved) f(t, v, j, integral_constant<bool, true>{});
        else f(t, v, j, integral_constant<bool, false>{});
    };
    auto type = [&](auto t) {
        integral_constant<int, 1> one;
        if (s.v == 8) {
            if constexpr (sizeof(t) == 2) near(t, integral_constant<int, 8>{}, one);
        } else if (s.v == 4) {
            near(t, integral_constant<int, 4>{}, one);
        } else if (s.j == 1) {
            near(t, one, one);
        } else {
            near(t, one, integral_constant<int, 4>{});
        }
    };
    if (d->dtype == IM2WIN_F32) type(float{});
    else type(bf16{});
}

QkArgs args_of(const im2win_qk_desc* d, const Shape& s, const void* q, const void* k, const float* wq, const float* wk, const int32_t* pos, const float* freqs) {
    QkArgs a{};
    a.q = q; a.k = k; a.wq = wq; a.wk = wk; a.pos = pos; a.freqs = freqs;
    a.ld_q = d->ld_q; a.ld_k = d->ld_k;
    a.tokens = (int)d->tokens; a.q_heads = (int)d->q_heads; a.k_heads = (int)d->k_heads; a.dim = (int)d->head_dim; a.rot = (int)d->rot_dim;
    a.lanes = s.lanes; a.parts = (int)s.parts;
    a.eps = d->eps; a.inv_d = 1.0f / (float)d->head_dim;
    // a side without heads is never read; its weights are loaded all the same
    if (!a.wq) a.wq = wk;
    if (!a.wk) a.wk = wq;
    return a;
}

int check_inputs(const im2win_qk_desc* d, const void* q, const void* k, const float* wq, const float* wk, const int32_t* pos, const float* freqs) {
    int rc;
    const size_t e = size_of(d->dtype);
    if (d->q_heads && ((rc = need_ptr(wq, 4, "wq")) || (d->tokens && (rc = need_ptr(q, e, "q"))))) return rc;
    if (d->k_heads && ((rc = need_ptr(wk, 4, "wk")) || (d->tokens && (rc = need_ptr(k, e, "k"))))) return rc;
    if (d->rot_dim && ((rc = need_ptr(freqs, 4, "freqs")) || (d->tokens && (rc = need_ptr(pos, 4, "positions"))))) return rc;
    return IM2WIN_OK;
}

}  // namespace
}  // namespace im2win

using namespace im2win;

extern "C" {

int im2win_qk_norm_rope(const im2win_qk_desc* d, const void* q, const void* k, const float* wq, const float* wk, const int32_t* positions,
                        const float* freqs, void* yq, void* yk, void* stream) {
    int rc = check_desc(d);
    if (rc || (rc = check_inputs(d, q, k, wq, wk, positions, freqs))) return rc;
    const size_t e = size_of(d->dtype);
    if (d->tokens && ((d->q_heads && (rc = need_ptr(yq, e, "yq"))) || (d->k_heads && (rc = need_ptr(yk, e, "yk"))))) return rc;
    if (d->tokens == 0) return ok();
    const Shape s = shape_of(d);
    if ((rc = check_launch(s.blocks, kWavesPer * kWave, "qk_norm_rope"))) return rc;
    QkArgs a = args_of(d, s, q, k, wq, wk, positions, freqs);
    a.yq = yq; a.yk = yk;
    with_shape(d, s, [&](auto t, auto v, auto j, auto near) {
        hipLaunchKernelGGL((qk_norm_rope_kernel<decltype(t), decltype(v)::value, decltype(j)::value, decltype(near)::value>),
                           dim3((unsigned)s.blocks), dim3(kWavesPer * kWave), 0, static_cast<hipStream_t>(stream), a);
    });
    return launched("qk_norm_rope");
}

int im2win_qk_norm_rope_backward_workspace_bytes(const im2win_qk_desc* d, size_t* bytes) {
    int rc = check_desc(d);
    if (rc) return rc;
    if (!bytes) return fail(IM2WIN_ENULL, "bytes is NULL");
    *bytes = (size_t)(bwd_blocks(shape_of(d), d->dtype) * 2 * d->head_dim * 4);
    return ok();
}

int im2win_qk_norm_rope_backward(const im2win_qk_desc* d, const void* dyq, const void* dyk, const void* q, const void* k, const float* wq,
                                 const float* wk, const int32_t* positions, const float* freqs, void* dq, void* dk, float* dwq, float* dwk,
                                 void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_desc(d);
    if (rc || (rc = check_inputs(d, q, k, wq, wk, positions, freqs)) || (rc = need_ptr(dwq, 4, "dwq")) || (rc = need_ptr(dwk, 4, "dwk"))) return rc;
    const size_t e = size_of(d->dtype);
    if (d->tokens && ((d->q_heads && ((rc = need_ptr(dyq, e, "dyq")) || (rc = need_ptr(dq, e, "dq")))) ||
                      (d->k_heads && ((rc = need_ptr(dyk, e, "dyk")) || (rc = need_ptr(dk, e, "dk")))) ||
                      (rc = need_ptr(workspace, 16, "workspace"))))
        return rc;
    const Shape s = shape_of(d);
    const int64_t blocks = bwd_blocks(s, d->dtype);
    const size_t need = (size_t)(blocks * 2 * d->head_dim * 4);
    if (workspace_bytes < need)
        return fail(IM2WIN_EWORKSPACE, "workspace holds %zu bytes, the gradients need %zu", workspace_bytes, need);
    hipStream_t st = static_cast<hipStream_t>(stream);
    QkArgs a = args_of(d, s, q, k, wq, wk, positions, freqs);
    a.dq = dyq; a.dk = dyk; a.yq = dq; a.yk = dk; a.part = static_cast<float*>(workspace);
    if (blocks)
        with_shape(d, s, [&](auto t, auto v, auto j, auto near) {
            hipLaunchKernelGGL((qk_norm_rope_bwd_kernel<decltype(t), decltype(v)::value, decltype(j)::value, decltype(near)::value>),
                               dim3((unsigned)blocks), dim3(kWavesPer * kWave), 0, st, a);
        });
    hipLaunchKernelGGL(qk_norm_rope_bwd_sum_kernel, dim3((unsigned)((2 * d->head_dim + kWave - 1) / kWave)), dim3(kSumWaves * kWave), 0, st,
                       a.part, dwq, dwk, (int)blocks, (int)d->head_dim);
    return launched("qk_norm_rope_backward");
}

}  // extern "C"
