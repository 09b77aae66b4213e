// Root-mean-square norm with the residual's addition (im2win_add_rms_norm*,
// include/im2win_seq.h).  One workgroup holds a row in registers, four or
// eight consecutive channels per thread and step: the row is read once, the squares
// are summed across lanes and waves, and the result leaves from registers.
// Bound by memory: 16384 x 4096 bf16 to 8 bits with a scale for each 128
// channels takes 87 us, 5.4 TB/s.  Workgroups of 256 threads and two steps beat
// one step of twice the threads (98 us) and four of half (97).
#include <algorithm>

#include "seq_common.h"

namespace im2win {
namespace {

// Consecutive channels of a thread and step: 16 bytes of the wider type, so
// that a wave's accesses of it have no gaps (10813 x 2176 fp32: 93 us with
// eight channels, 83 with four); eight where the output is 8 bits, whose
// scales belong to neighbouring lanes.
template <typename TX, typename TR, bool FP8>
constexpr int kChannels = FP8 || (sizeof(TX) == 2 && sizeof(TR) == 2) ? 8 : 4;
constexpr int kPer = 8;   // channels of a thread and of a step of eight, by which workgroups are shaped

struct NormArgs {
    const void* x;
    const void* res;
    const float* w;
    void* y;
    float* scales;
    void* h;
    int64_t ld_x;
    int channels;
    int block;     // channels per scale, 0: the row
    float eps;
    float inv_d;
};

// N consecutive elements of which the first `n` exist, as they lie in memory:
// whole at any address, and element by element for the last thread of a row
// whose channels are no multiple of N.  get() converts, so that the loads of
// several arrays are in flight together.
template <typename T, int N>
struct Run {
    static constexpr int kWords = N * (int)sizeof(T) / 4;
    uint32_t u[kWords];

    static constexpr int kPiece = kWords < 4 ? kWords : 4;      // one access
    __device__ __forceinline__ void load(const T* p) {
#pragma unroll
        for (int i = 0; i < kWords; i += kPiece) __builtin_memcpy(u + i, reinterpret_cast<const char*>(p) + 4 * i, 4 * kPiece);
    }
    __device__ __forceinline__ void load(const T* p, int n) {
        T e[N];
#pragma unroll
        for (int i = 0; i < N; ++i) e[i] = i < n ? p[i] : (T)0.0f;
        __builtin_memcpy(u, e, sizeof u);
    }
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int i = 0; i < kWords; ++i) u[i] = 0;
    }
    __device__ __forceinline__ float get(int i) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(u[i]);
        else return __uint_as_float(i % 2 ? u[i / 2] & 0xffff0000u : u[i / 2] << 16);
    }
};

// The same N channels of up to three arrays
template <int N, typename A, typename B, typename C>
__device__ __forceinline__ void load_runs(int n, Run<A, N>& a, const A* pa, Run<B, N>& b, const B* pb, Run<C, N>& c, const C* pc, bool have_c) {
    a.zero();
    b.zero();
    c.zero();
    if (n >= N) {
        a.load(pa);
        b.load(pb);
        if (have_c) c.load(pc);
    } else if (n > 0) {
        a.load(pa, n);
        b.load(pb, n);
        if (have_c) c.load(pc, n);
    }
}

template <typename T, int N>
__device__ __forceinline__ void put_run(T* p, int n, const float (&v)[N]) {
    if (n >= N) {
        if constexpr (N == kVec<T> || N == 2 * kVec<T>) {
            store_run<N>(p, v);
        } else {
            static_assert(N == 4 && sizeof(T) == 2, "half a vector");
            const uint32_t w[2] = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
            __builtin_memcpy(p, w, 8);
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < n) p[i] = (T)v[i];
    }
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int m = 1; m < kWave; m *= 2) v += __shfl_xor(v, m);
    return v;
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
#pragma unroll
    for (int m = 1; m < kWave; m *= 2) v = max(v, (uint32_t)__shfl_xor((int)v, m));
    return v;
}

// Sum or maximum over the workgroup's NT threads, the waves' values in order.
// `part` holds NT / 64 values; the caller keeps a barrier between two uses.
template <int NT>
__device__ __forceinline__ float block_sum(float v, float* part) {
    v = wave_sum(v);
    if constexpr (NT > kWave) {
        if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = v;
        __syncthreads();
        v = part[0];
#pragma unroll
        for (int i = 1; i < NT / kWave; ++i) v += part[i];
    }
    return v;
}
template <int NT>
__device__ __forceinline__ uint32_t block_max(uint32_t v, uint32_t* part) {
    v = wave_max(v);
    if constexpr (NT > kWave) {
        if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = v;
        __syncthreads();
        v = part[0];
#pragma unroll
        for (int i = 1; i < NT / kWave; ++i) v = max(v, part[i]);
    }
    return v;
}

// Four fp32 values as e4m3 bytes, rounded to nearest even: |v| is at most 448
// and one rounding of the division, which rounds to 448.  Anything farther
// beyond 448 becomes NaN.
__device__ __forceinline__ uint32_t pack_fp8(float a, float b, float c, float d) {
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
}

constexpr float kSmallestNormal = 0x1p-126f;

// TX: x and y.  TR: residual and h.  NT threads, STEPS times eight channels
// per thread (NT * STEPS * 8 >= channels).
template <typename TX, typename TR, int NT, int STEPS, bool FP8>
__global__ __launch_bounds__(NT) void add_rms_norm_kernel(NormArgs a) {
    constexpr int N = kChannels<TX, TR, FP8>, NV = STEPS * kPer / N;
    __shared__ float part[NT / kWave];
    __shared__ uint32_t top_part[NT / kWave];
    const int64_t row = blockIdx.x;
    const TX* x = static_cast<const TX*>(a.x) + row * a.ld_x;
    const TR* res = static_cast<const TR*>(a.res) + row * a.channels;
    TR* h = static_cast<TR*>(a.h) + row * a.channels;
    Run<TX, N> xr[NV];
    Run<float, N> w[NV];
    Run<TR, N> rr[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int c = (j * NT + (int)threadIdx.x) * N;
        load_runs<N>(a.channels - c, xr[j], x + c, w[j], a.w + c, rr[j], res + c, a.res != nullptr);
    }
    float v[NV][N];
    float ss = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int c = (j * NT + (int)threadIdx.x) * N, n = a.channels - c;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[j][i] = xr[j].get(i) + rr[j].get(i);
            if constexpr (sizeof(TR) == 2) v[j][i] = (float)(TR)v[j][i];   // the norm is that of h as it is kept
            ss = fmaf(v[j][i], v[j][i], ss);
        }
        if (a.h && n > 0) put_run(h + c, n, v[j]);
    }
    const float r = 1.0f / sqrtf(fmaf(block_sum<NT>(ss, part), a.inv_d, a.eps));
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < N; ++i) v[j][i] = v[j][i] * r * w[j].get(i);

    if constexpr (!FP8) {
        TX* y = static_cast<TX*>(a.y) + row * a.channels;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * NT + (int)threadIdx.x) * N, n = a.channels - c;
            if (n > 0) put_run(y + c, n, v[j]);
        }
    } else {
        uint8_t* q = static_cast<uint8_t*>(a.y) + row * a.channels;
        // magnitudes as integers: their order is the floats', and a NaN is above them all
        uint32_t top[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            top[j] = 0;
#pragma unroll
            for (int i = 0; i < N; ++i) top[j] = max(top[j], __float_as_uint(v[j][i]) & 0x7fffffffu);
        }
        if (a.block == 0) {
            uint32_t m = top[0];
#pragma unroll
            for (int j = 1; j < NV; ++j) m = max(m, top[j]);
            m = block_max<NT>(m, top_part);
#pragma unroll
            for (int j = 0; j < NV; ++j) top[j] = m;
        } else {
            // block / 8 neighbouring lanes share a scale (the block is a power of two up to 512)
#pragma unroll
            for (int j = 0; j < NV; ++j)
                for (int m = 1; m < a.block / N; m *= 2) top[j] = max(top[j], (uint32_t)__shfl_xor((int)top[j], m));
        }
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * NT + (int)threadIdx.x) * N, n = a.channels - c;
            if (n <= 0) continue;
            const float most = __uint_as_float(top[j]);
            const float share = most / 448.0f;
            const float scale = share > 0.0f ? share : 1.0f;     // it may round to 0, and is NaN beside a NaN
            if (a.block == 0) {
                if (c == 0) a.scales[row] = scale;
            } else if (c % a.block == 0) {
                a.scales[row * (a.channels / a.block) + c / a.block] = scale;
            }
            float s[N];
#pragma unroll
            for (int i = 0; i < N; ++i) s[i] = v[j][i] / scale;
            // a subnormal scale has few bits, so that it may be too small for its block by up to a third
            if (scale < kSmallestNormal)
#pragma unroll
                for (int i = 0; i < N; ++i) s[i] = fminf(fmaxf(s[i], -448.0f), 448.0f);
            const uint32_t lo = pack_fp8(s[0], s[1], s[2], s[3]), hi = pack_fp8(s[4], s[5], s[6], s[7]);
            if (n >= N) {
                const uint32_t both[2] = {lo, hi};
                __builtin_memcpy(q + c, both, 8);
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i)
                    if (i < n) q[c + i] = (uint8_t)((i < 4 ? lo : hi) >> (8 * (i % 4)));
            }
        }
    }
}

// ---------------------------------------------------------------------------
// Gradients: each workgroup walks rows row0, row0 + gridDim.x, ... with its
// part of dw in registers, and leaves one row of partial sums; a second
// kernel adds those in order.  Bound by memory: 16384 x 4096 bf16 takes 107 us,
// 5.0 TB/s; 8191 x 2049 with a residual in fp32 58 us, 4.1 TB/s.
// ---------------------------------------------------------------------------
struct NormBwdArgs {
    const void* dy;
    const void* h;
    const float* w;
    const void* dres;
    void* dx;
    float* part;     // [blocks][channels]
    float* dw;
    int tokens;
    int channels;
    int blocks;
    float eps;
    float inv_d;
};

template <typename TX, typename TR, int NT, int STEPS>
__global__ __launch_bounds__(NT) void add_rms_norm_bwd_kernel(NormBwdArgs a) {
    constexpr int N = kChannels<TX, TR, false>, NV = STEPS * kPer / N;
    __shared__ float part[2][2][NT / kWave];
    float dw[NV][N] = {};
    int turn = 0;
    for (int64_t row = blockIdx.x; row < a.tokens; row += gridDim.x, turn ^= 1) {
        const TX* dy = static_cast<const TX*>(a.dy) + row * a.channels;
        const TR* h = static_cast<const TR*>(a.h) + row * a.channels;
        const TR* dres = static_cast<const TR*>(a.dres) + row * a.channels;
        Run<TX, N> g[NV];
        Run<float, N> w[NV];
        Run<TR, N> v[NV], d0[NV];
        float ss = 0.0f, gh = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * NT + (int)threadIdx.x) * N;
            load_runs<N>(a.channels - c, g[j], dy + c, v[j], h + c, d0[j], dres + c, a.dres != nullptr);
        }
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * NT + (int)threadIdx.x) * N;
            Run<float, N> none;
            load_runs<N>(a.channels - c, w[j], a.w + c, none, a.w + c, none, a.w, false);
        }
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                ss = fmaf(v[j].get(i), v[j].get(i), ss);
                gh = fmaf(g[j].get(i) * w[j].get(i), v[j].get(i), gh);
            }
        // two arrays of partial sums in turn: a wave that is a row ahead writes the other one, and
        // it cannot be two ahead, as every row has a barrier
        ss = wave_sum(ss);
        gh = wave_sum(gh);
        if constexpr (NT > kWave) {
            if (threadIdx.x % kWave == 0) {
                part[turn][0][threadIdx.x / kWave] = ss;
                part[turn][1][threadIdx.x / kWave] = gh;
            }
            __syncthreads();
            ss = part[turn][0][0];
            gh = part[turn][1][0];
#pragma unroll
            for (int i = 1; i < NT / kWave; ++i) {
                ss += part[turn][0][i];
                gh += part[turn][1][i];
            }
        }
        const float r = 1.0f / sqrtf(fmaf(ss, a.inv_d, a.eps));
        const float k = r * r * gh * a.inv_d;
        TR* dx = static_cast<TR*>(a.dx) + row * a.channels;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * NT + (int)threadIdx.x) * N, n = a.channels - c;
            float d[N];
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float gi = g[j].get(i), hi = v[j].get(i);
                d[i] = fmaf(r, fmaf(-k, hi, gi * w[j].get(i)), d0[j].get(i));
                dw[j][i] = fmaf(gi * r, hi, dw[j][i]);
            }
            if (n > 0) put_run(dx + c, n, d);
        }
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int c = (j * NT + (int)threadIdx.x) * N, n = a.channels - c;
        if (n > 0) put_run(a.part + (int64_t)blockIdx.x * a.channels + c, n, dw[j]);
    }
}

constexpr int kSumWaves = 16;

// dw from the workgroups' sums: 64 channels per workgroup, every 16th row per
// wave, eight rows' loads in flight
__global__ __launch_bounds__(kSumWaves * kWave) void add_rms_norm_bwd_sum_kernel(NormBwdArgs a) {
    __shared__ float sum[kSumWaves][kWave];
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    const int c = (int)blockIdx.x * kWave + lane;
    float s = 0.0f;
    if (c < a.channels) {
#pragma unroll 8
        for (int i = wave; i < a.blocks; i += kSumWaves) s += a.part[(int64_t)i * a.channels + c];
    }
    sum[wave][lane] = s;
    __syncthreads();
    if (wave == 0 && c < a.channels) {
        for (int i = 1; i < kSumWaves; ++i) s += sum[i][lane];
        a.dw[c] = s;
    }
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
constexpr int64_t kMaxNormChannels = 16384;

// Workgroups of the gradients: enough rows in flight to fill the chip, few
// enough that the partial sums stay a small part of the traffic.
int64_t bwd_blocks(int64_t tokens) { return tokens < 1024 ? tokens : 1024; }

int check_desc(const im2win_norm_desc* d) {
    if (!d) return fail(IM2WIN_ENULL, "descriptor is NULL");
    int rc = check_rows(d->tokens, d->channels, d->dtype);
    if (rc) return rc;
    if (d->residual_dtype != IM2WIN_F32 && d->residual_dtype != IM2WIN_BF16)
        return fail(IM2WIN_EINVAL, "unknown residual dtype %d", (int)d->residual_dtype);
    if (d->channels > kMaxNormChannels)
        return fail(IM2WIN_EOVERFLOW, "the norm holds rows of at most %lld channels (got %lld)",
                    (long long)kMaxNormChannels, (long long)d->channels);
    if (!(d->eps >= 0.0f)) return fail(IM2WIN_EINVAL, "eps must be >= 0 (got %g)", (double)d->eps);
    if (d->block && (d->block < 16 || d->block > 512 || (d->block & (d->block - 1)) || d->channels % d->block))
        return fail(IM2WIN_EINVAL, "block must be 0 or a power of two from 16 to 512 that divides the %lld channels (got %lld)",
                    (long long)d->channels, (long long)d->block);
    return check_ld(d->ld_x, d->channels, "ld_x");
}

size_t size_of(int32_t dtype) { return dtype == IM2WIN_F32 ? 4 : 2; }

// f(threads, steps): the smallest workgroup that holds the row.  A wave per
// row up to 512 channels, then 256 threads of one to four steps, then 1024
// of two: 16384 channels, which their 128 registers just hold beside dw (the
// gradients spill one of them in fp32, five with a bf16 dy and fp32 rows).
template <typename F>
void with_shape(int64_t channels, F f) {
    using std::integral_constant;
    if (channels <= 64 * kPer) f(integral_constant<int, 64>{}, integral_constant<int, 1>{});
    else if (channels <= 256 * kPer) f(integral_constant<int, 256>{}, integral_constant<int, 1>{});
    else if (channels <= 512 * kPer) f(integral_constant<int, 256>{}, integral_constant<int, 2>{});
    else if (channels <= 1024 * kPer) f(integral_constant<int, 256>{}, integral_constant<int, 4>{});
    else f(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
}

template <typename F>
void with_types(const im2win_norm_desc* d, F f) {
    if (d->dtype == IM2WIN_F32) {
        if (d->residual_dtype == IM2WIN_F32) f(float{}, float{});
        else f(float{}, bf16{});
    } else {
        if (d->residual_dtype == IM2WIN_F32) f(bf16{}, float{});
        else f(bf16{}, bf16{});
    }
}

template <bool FP8>
int forward(const im2win_norm_desc* d, const void* x, const void* residual, const float* w, void* y, float* scales,
            void* h, void* stream) {
    int rc = check_desc(d);
    if (rc) return rc;
    if (!FP8 && d->block) return fail(IM2WIN_EINVAL, "block (%lld) is for the 8-bit output", (long long)d->block);
    if ((rc = need_ptr(w, 4, "w"))) return rc;
    if (d->tokens == 0) return ok();
    const size_t ex = size_of(d->dtype), er = size_of(d->residual_dtype);
    if ((rc = need_ptr(x, ex, "x")) || (rc = may_ptr(residual, er, "residual")) ||
        (rc = need_ptr(y, FP8 ? 1 : ex, FP8 ? "q" : "y")) || (rc = may_ptr(h, er, "h")))
        return rc;
    if (FP8 && (rc = need_ptr(scales, 4, "scales"))) return rc;
    if (residual && !h) return fail(IM2WIN_ENULL, "h is NULL (it may be the residual itself)");
    NormArgs a{};
    a.w = w;
    a.ld_x = d->ld_x; a.channels = (int)d->channels; a.block = (int)d->block;
    a.eps = d->eps; a.inv_d = 1.0f / (float)d->channels;
    with_types(d, [&](auto tx, auto tr) {
        with_shape(d->channels, [&](auto nt, auto nv) {
            using TX = decltype(tx);
            using TR = decltype(tr);
            constexpr int NT = decltype(nt)::value, NV = decltype(nv)::value;
            // a workgroup a row: from 2^22 rows (of 1024 threads) to 2^26 (of 64) a launch holds no more
            constexpr int64_t kMost = kMaxThreads / NT;
            for (int64_t first = 0; first < d->tokens; first += kMost) {
                const int64_t rows = std::min(kMost, d->tokens - first), at = first * d->channels;
                a.x = static_cast<const TX*>(x) + first * d->ld_x;
                a.res = residual ? static_cast<const TR*>(residual) + at : nullptr;
                a.h = h ? static_cast<TR*>(h) + at : nullptr;
                if constexpr (FP8) {
                    a.y = static_cast<uint8_t*>(y) + at;
                    a.scales = scales + (d->block ? at / d->block : first);
                } else {
                    a.y = static_cast<TX*>(y) + at;
                }
                hipLaunchKernelGGL((add_rms_norm_kernel<TX, TR, NT, NV, FP8>), dim3((unsigned)rows), dim3(NT), 0,
                                   static_cast<hipStream_t>(stream), a);
            }
        });
    });
    return launched(FP8 ? "add_rms_norm_fp8" : "add_rms_norm");
}

}  // namespace
}  // namespace im2win

using namespace im2win;

extern "C" {

int im2win_add_rms_norm(const im2win_norm_desc* d, const void* x, const void* residual, const float* w, void* y,
                        void* h, void* stream) {
    return forward<false>(d, x, residual, w, y, nullptr, h, stream);
}

int im2win_add_rms_norm_fp8(const im2win_norm_desc* d, const void* x, const void* residual, const float* w, void* q,
                            float* scales, void* h, void* stream) {
    return forward<true>(d, x, residual, w, q, scales, h, stream);
}

int im2win_add_rms_norm_backward_workspace_bytes(const im2win_norm_desc* d, size_t* bytes) {
    int rc = check_desc(d);
    if (rc) return rc;
    if (!bytes) return fail(IM2WIN_ENULL, "bytes is NULL");
    *bytes = (size_t)(bwd_blocks(d->tokens) * d->channels * 4);
    return ok();
}

int im2win_add_rms_norm_backward(const im2win_norm_desc* d, const void* dy, const void* h, const float* w,
                                 const void* d_residual, void* dx, float* dw, void* workspace,
                                 size_t workspace_bytes, void* stream) {
    int rc = check_desc(d);
    if (rc || (rc = need_ptr(w, 4, "w")) || (rc = need_ptr(dw, 4, "dw"))) return rc;
    const size_t ex = size_of(d->dtype), er = size_of(d->residual_dtype);
    const int64_t blocks = bwd_blocks(d->tokens);
    if (d->tokens && ((rc = need_ptr(dy, ex, "dy")) || (rc = need_ptr(h, er, "h")) || (rc = need_ptr(dx, er, "dx")) ||
                      (rc = may_ptr(d_residual, er, "d_residual")) || (rc = need_ptr(workspace, 16, "workspace"))))
        return rc;
    const size_t need = (size_t)(blocks * d->channels * 4);
    if (workspace_bytes < need)
        return fail(IM2WIN_EWORKSPACE, "workspace holds %zu bytes, the gradients need %zu", workspace_bytes, need);
    NormBwdArgs a{};
    a.dy = dy; a.h = h; a.w = w; a.dres = d_residual; a.dx = dx; a.part = static_cast<float*>(workspace); a.dw = dw;
    a.tokens = (int)d->tokens; a.channels = (int)d->channels; a.blocks = (int)blocks;
    a.eps = d->eps; a.inv_d = 1.0f / (float)d->channels;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (blocks)
        with_types(d, [&](auto tx, auto tr) {
            with_shape(d->channels, [&](auto nt, auto nv) {
                using TX = decltype(tx);
                using TR = decltype(tr);
                constexpr int NT = decltype(nt)::value, NV = decltype(nv)::value;
                hipLaunchKernelGGL((add_rms_norm_bwd_kernel<TX, TR, NT, NV>),
                                   dim3((unsigned)blocks), dim3(NT), 0, s, a);
            });
        });
    hipLaunchKernelGGL(add_rms_norm_bwd_sum_kernel, dim3((unsigned)((d->channels + kWave - 1) / kWave)),
                       dim3(kSumWaves * kWave), 0, s, a);
    return launched("add_rms_norm_backward");
}

}  // extern "C"
