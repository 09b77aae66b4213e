// The selective scan's layout, shared by its forward and backward kernels.
//
// Four neighbouring lanes (a quad) share CH neighbouring channels and hold a
// quarter of their N states each, NS = ceil(N / 4) rounded up to a compiled
// size, in registers; a wave covers 16*CH channels and walks the rows of its
// chunk of tokens.  What is needed once for a row and channel (the step size,
// x, the gate) is computed for four rows at a time, one row per lane of the
// quad, and passed around by lane permutations; sums over the states are
// sums over the quad.  B and C of a tile of rows are staged in LDS as fp32
// for the four waves of a workgroup.
#pragma once

#include "seq_common.h"

namespace im2win {

constexpr float kLog2e = 1.44269504088896f;
constexpr int kQuad = 4;
constexpr int kScanWaves = 4;
constexpr int kScanTile = 32;     // rows whose B and C lie in LDS

struct ScanArgs {
    const void* x;
    const void* dt;
    const float* A;
    const void* B;
    const void* C;
    const float* D;
    const void* z;
    const float* dt_bias;
    const float* init;
    void* y;
    float* final_state;
    SeqMap seq;
    int64_t ld_x, ld_dt, ld_z, ld_b, ld_c;
    int channels;
    int states;
    int group_channels;    // D / G
    int group_blocks;      // workgroups that cover a group's channels
    int blocks;            // G * group_blocks
    int chunk;             // rows per chunk
    int chunks;
    int softplus;
    int wide;              // rows of pairs of channels can be read and written in one access
    float* carry;          // [chunks][channels][4*NS]: the state behind each chunk
    float* span;           // [chunks][channels]: the sum of step sizes that the state passes
    int* flags;            // [chunks]
};

// flags: the chunk's last sequence goes on behind it / began inside it
constexpr int kGoesOn = 1, kBegan = 2;

template <int J>
__device__ __forceinline__ float quad_get(float v) {   // the value of the quad's lane J
    return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), J * 0x55, 0xf, 0xf, true));
}
__device__ __forceinline__ float quad_sum(float v) {   // in every lane of the quad
    v += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0xB1, 0xf, 0xf, true));   // lanes 1 0 3 2
    v += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x4E, 0xf, 0xf, true));   // lanes 2 3 0 1
    return v;
}

// log(1 + exp(v)) = max(v, 0) + log1p(e), e = exp(-|v|), and log1p(e) =
// 2 atanh(s) with s = e / (2 + e) <= 1/3 by its power series, whose first
// term left out is s^17 / 17 < 1e-9: small steps keep their relative accuracy.
__device__ __forceinline__ float softplus(float v) {
    const float e = __builtin_amdgcn_exp2f(-kLog2e * fabsf(v));
    const float s = e * __builtin_amdgcn_rcpf(2.0f + e), q = s * s;
    float p = 1.0f / 15.0f;
    p = fmaf(p, q, 1.0f / 13.0f);
    p = fmaf(p, q, 1.0f / 11.0f);
    p = fmaf(p, q, 1.0f / 9.0f);
    p = fmaf(p, q, 1.0f / 7.0f);
    p = fmaf(p, q, 1.0f / 5.0f);
    p = fmaf(p, q, 1.0f / 3.0f);
    return fmaxf(v, 0.0f) + fmaf(2.0f * s * q, p, 2.0f * s);
}

// CH neighbouring channels of a row as they lie in memory; the conversion is
// left to get(), so that a load can stay in flight.  `wide`: one access.
template <typename T, int CH> struct Raw;

template <> struct Raw<float, 1> {
    float v;
    __device__ __forceinline__ void load(const float* row, const int (&c)[1], bool) { v = row[c[0]]; }
    __device__ __forceinline__ float get(int, bool) const { return v; }
};
template <> struct Raw<float, 2> {
    float2 v;
    __device__ __forceinline__ void load(const float* row, const int (&c)[2], bool wide) {
        if (wide) v = *reinterpret_cast<const float2*>(row + c[0]);
        else v = make_float2(row[c[0]], row[c[1]]);
    }
    __device__ __forceinline__ float get(int i, bool) const { return i ? v.y : v.x; }
};
template <> struct Raw<bf16, 1> {
    uint16_t v;
    __device__ __forceinline__ void load(const bf16* row, const int (&c)[1], bool) {
        v = reinterpret_cast<const uint16_t*>(row)[c[0]];
    }
    __device__ __forceinline__ float get(int, bool) const { return __uint_as_float((uint32_t)v << 16); }
};
template <> struct Raw<bf16, 2> {
    uint32_t a, b;     // both channels in a where wide, one in each otherwise
    __device__ __forceinline__ void load(const bf16* row, const int (&c)[2], bool wide) {
        const uint16_t* p = reinterpret_cast<const uint16_t*>(row);
        if (wide) {
            a = *reinterpret_cast<const uint32_t*>(p + c[0]);
        } else {
            a = p[c[0]];
            b = p[c[1]];
        }
    }
    __device__ __forceinline__ float get(int i, bool wide) const {
        return __uint_as_float(i == 0 ? a << 16 : wide ? a & 0xffff0000u : b << 16);
    }
};

template <int CH>
__device__ __forceinline__ void store_channels(float* row, int c, const bool (&live)[CH], const float (&v)[CH], bool wide) {
    if constexpr (CH == 2) {
        if (wide) {
            if (live[0]) *reinterpret_cast<float2*>(row + c) = make_float2(v[0], v[1]);
            return;
        }
    }
#pragma unroll
    for (int i = 0; i < CH; ++i)
        if (live[i]) row[c + i] = v[i];
}
template <int CH>
__device__ __forceinline__ void store_channels(bf16* row, int c, const bool (&live)[CH], const float (&v)[CH], bool wide) {
    if constexpr (CH == 2) {
        if (wide) {
            if (live[0]) *reinterpret_cast<uint32_t*>(row + c) = pack_bf16(v[0], v[1]);
            return;
        }
    }
#pragma unroll
    for (int i = 0; i < CH; ++i)
        if (live[i]) row[c + i] = (bf16)v[i];
}

// NS consecutive floats of LDS on a boundary of their largest power of two
template <int NS>
__device__ __forceinline__ void lds_row(const float* p, float (&v)[NS]) {
    if constexpr (NS % 4 == 0) {
#pragma unroll
        for (int i = 0; i < NS; i += 4) {
            const float4 f = *reinterpret_cast<const float4*>(p + i);
            v[i] = f.x; v[i + 1] = f.y; v[i + 2] = f.z; v[i + 3] = f.w;
        }
    } else if constexpr (NS % 2 == 0) {
#pragma unroll
        for (int i = 0; i < NS; i += 2) {
            const float2 f = *reinterpret_cast<const float2*>(p + i);
            v[i] = f.x; v[i + 1] = f.y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < NS; ++i) v[i] = p[i];
    }
}

// The channels of a lane
template <int CH>
struct Lane {
    int q;              // lane of the quad: its quarter of the states, and its row of four
    int c0;             // first channel (may lie past the group)
    int c[CH];          // channels to read from: past the group, its first one
    bool live[CH];

    __device__ __forceinline__ void init(const ScanArgs& a, int block, int wave) {
        const int lane = threadIdx.x % kWave;
        q = lane % kQuad;
        const int group = block / a.group_blocks;
        const int from = group * a.group_channels, to = from + a.group_channels;
        c0 = from + ((block % a.group_blocks) * kScanWaves + wave) * (kWave / kQuad) * CH + lane / kQuad * CH;
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            live[i] = c0 + i < to;
            c[i] = live[i] ? c0 + i : from + (a.wide ? i : 0);
        }
    }
};

// B or C of rows [t, t + n), n <= kScanTile, as fp32; states past N and rows past n are zero
template <typename T, int NS>
__device__ __forceinline__ void stage(float* lds, const T* m, int64_t ld, int group_offset, int states, int t, int n) {
    constexpr int NP = kQuad * NS;
    for (int i = threadIdx.x; i < kScanTile * NP; i += kScanWaves * kWave) {
        const int r = i / NP, s = i % NP;
        lds[i] = r < n && s < states ? (float)m[(int64_t)(t + r) * ld + group_offset + s] : 0.0f;
    }
}

// Compiled shapes: f(NS, CH) for N states
template <typename F>
void with_states(int64_t n, F f) {
    using std::integral_constant;
    if (n <= 8) f(integral_constant<int, 2>{}, integral_constant<int, 2>{});
    else if (n <= 16) f(integral_constant<int, 4>{}, integral_constant<int, 2>{});
    else if (n <= 24) f(integral_constant<int, 6>{}, integral_constant<int, 2>{});
    else if (n <= 32) f(integral_constant<int, 8>{}, integral_constant<int, 1>{});
    else if (n <= 64) f(integral_constant<int, 16>{}, integral_constant<int, 1>{});
    else f(integral_constant<int, 32>{}, integral_constant<int, 1>{});
}

// Checks and geometry that the entry points share (seq_scan.hip)
int check_scan(const im2win_scan_desc* d, bool sequences, const int32_t* starts, bool have_starts);
int check_scan_inputs(const im2win_scan_desc* d, const void* x, const void* dt, const float* A, const void* B,
                      const void* C, const float* D, const void* z, const float* dt_bias);
ScanArgs scan_args(const im2win_scan_desc* d, const void* x, const void* dt, const float* A, const void* B,
                   const void* C, const float* D, const void* z, const float* dt_bias, int ch);

}  // namespace im2win
