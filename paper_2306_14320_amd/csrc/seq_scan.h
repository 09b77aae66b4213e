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
    float* carry;          // [chunks][channels][4*NS]: the state behind each chunk
    float* span;           // [chunks][channels]: the sum of step sizes that the state passes
    int* flags;            // [chunks]
    int look;              // no carry kernel runs: carry holds the chunks' own states (see carried)
};

// flags of a chunk: its last sequence goes on behind it / its first sequence
// began before it / both of one sequence that fills the chunk
constexpr int kGoesOn = 1, kFromBefore = 2, kThrough = 4;

template <int J>
__device__ __forceinline__ float quad_get(float v) {   // the value of the quad's lane J
    return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), J * 0x55, 0xf, 0xf, true));
}
__device__ __forceinline__ float quad_sum(float v) {   // in every lane of the quad
    v += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0xB1, 0xf, 0xf, true));   // lanes 1 0 3 2
    v += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x4E, 0xf, 0xf, true));   // lanes 2 3 0 1
    return v;
}

// Four rows' values, each spread over the quad's lanes, summed: lane J gets row J's.
__device__ __forceinline__ float quad_sums(float r0, float r1, float r2, float r3, int q) {
    auto cross = [](float own, float other, auto lanes) {
        return own + __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(other), decltype(lanes)::value, 0xf, 0xf, true));
    };
    using std::integral_constant;
    const bool odd = q & 1, high = q & 2;
    const float low = cross(odd ? r1 : r0, odd ? r0 : r1, integral_constant<int, 0xB1>{});
    const float top = cross(odd ? r3 : r2, odd ? r2 : r3, integral_constant<int, 0xB1>{});
    return cross(high ? top : low, high ? low : top, integral_constant<int, 0x4E>{});
}

// log(1 + exp(v)) = max(v, 0) + log1p(e), e = exp(-|v|), and log1p(e) =
// 2 atanh(s) with s = e / (2 + e) <= 1/3.  atanh(s) / s is a polynomial in q =
// s^2 <= 1/9, interpolated at the Chebyshev nodes of that interval to 4e-9:
// small steps keep their relative accuracy.
__device__ __forceinline__ float softplus(float v) {
    const float e = __builtin_amdgcn_exp2f(-kLog2e * fabsf(v));
    const float s = e * __builtin_amdgcn_rcpf(2.0f + e), q = s * s;
    float p = 0.140873286f;
    p = fmaf(p, q, 0.139807094f);
    p = fmaf(p, q, 0.200124269f);
    p = fmaf(p, q, 0.33333158f);
    return fmaxf(v, 0.0f) + fmaf(2.0f * s * q, p, 2.0f * s);
}

// Device memory by its address space, which a pointer pinned to registers keeps
// only where its type says so; the words' types have an element's alignment.
#define IM2WIN_GLOBAL __attribute__((address_space(1)))
using GlobalIn = const IM2WIN_GLOBAL char*;
using GlobalOut = IM2WIN_GLOBAL char*;
typedef uint16_t Word16;
typedef uint32_t Word32 __attribute__((aligned(2)));
typedef uint32_t Word64 __attribute__((ext_vector_type(2), aligned(4)));

// CH neighbouring channels of a row as they lie in memory, one access at any
// address; the conversion is left to get(), so that a load can stay in flight.
template <typename T, int CH>
struct Raw {
    static_assert(CH == 1 || CH == 2, "one channel or two");
    static constexpr int kBytes = CH * (int)sizeof(T), kWords = (kBytes + 3) / 4;
    uint32_t u[kWords];
    __device__ __forceinline__ void load(GlobalIn p) {
        if constexpr (kBytes == 2) {
            u[0] = *reinterpret_cast<const IM2WIN_GLOBAL Word16*>(p);
        } else if constexpr (kBytes == 4) {
            u[0] = *reinterpret_cast<const IM2WIN_GLOBAL Word32*>(p);
        } else {
            const Word64 v = *reinterpret_cast<const IM2WIN_GLOBAL Word64*>(p);
            u[0] = v.x;
            u[kWords - 1] = v.y;
        }
    }
    __device__ __forceinline__ float get(int i) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(u[i]);
        else return __uint_as_float(i ? u[0] & 0xffff0000u : u[0] << 16);
    }
    __device__ __forceinline__ void wait() {
#pragma unroll
        for (int i = 0; i < kWords; ++i) arrive(u[i]);
    }
};

// The channels of a row that a lane owns
__device__ __forceinline__ void store_one(GlobalOut p, float v, float) { *reinterpret_cast<IM2WIN_GLOBAL float*>(p) = v; }
__device__ __forceinline__ void store_one(GlobalOut p, float v, bf16) {
    *reinterpret_cast<IM2WIN_GLOBAL Word16*>(p) = __builtin_bit_cast(uint16_t, (bf16)v);
}
template <typename T, int CH>
__device__ __forceinline__ void store_channels(GlobalOut p, const bool (&live)[CH], const float (&v)[CH]) {
    if constexpr (CH == 2) {
        if (live[0] && live[1]) {
            if constexpr (sizeof(T) == 4) {
                const Word64 w = {__float_as_uint(v[0]), __float_as_uint(v[1])};
                *reinterpret_cast<IM2WIN_GLOBAL Word64*>(p) = w;
            } else {
                *reinterpret_cast<IM2WIN_GLOBAL Word32*>(p) = pack_bf16(v[0], v[1]);
            }
            return;
        }
    }
#pragma unroll
    for (int i = 0; i < CH; ++i)
        if (live[i]) store_one(p + i * (int)sizeof(T), v[i], T{});
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

// The channels of a lane: c to c + CH - 1.  A lane past its group, and the
// second place of a group's odd last channel, hold other channels of the row
// (whose memory exists) and are not live; the last channel of a row of them is
// the second place of the pair in front of it.
template <int CH>
struct Lane {
    int q;              // lane of the quad: its quarter of the states, and its row of four
    int c;
    bool live[CH];

    __device__ __forceinline__ void init(const ScanArgs& a, int block, int wave) {
        const int lane = threadIdx.x % kWave;
        q = lane % kQuad;
        const int group = block / a.group_blocks;
        const int from = group * a.group_channels, to = from + a.group_channels;
        const int own = from + ((block % a.group_blocks) * kScanWaves + wave) * (kWave / kQuad) * CH + lane / kQuad * CH;
        c = min(own, a.channels - CH);
#pragma unroll
        for (int i = 0; i < CH; ++i) live[i] = c + i >= own && c + i < to;
    }
};

// A T x D array: the rows of a group of four, one for each lane of the quad.
// The group's first row is a scalar address (pinned to scalar registers) and a
// lane's place beside it a 32-bit offset, so that a group costs no vector
// instruction for addresses.
template <typename T>
struct RowPlace {
    uint32_t offset;
    template <int CH>
    __device__ __forceinline__ RowPlace(int64_t ld, const Lane<CH>& l, int row) : offset((uint32_t)((row * ld + l.c) * (int64_t)sizeof(T))) {}
    __device__ __forceinline__ GlobalIn at(const void* m, int64_t ld, int t) const {
        GlobalIn base = (GlobalIn)m + t * ld * (int64_t)sizeof(T);
        asm("" : "+s"(base));
        return base + offset;
    }
    __device__ __forceinline__ GlobalOut at(void* m, int64_t ld, int t) const {
        GlobalOut base = (GlobalOut)m + t * ld * (int64_t)sizeof(T);
        asm("" : "+s"(base));
        return base + offset;
    }
};

// A lane's quarter of the N floats at m; states past N are zero
template <int NS>
__device__ __forceinline__ void load_states(const float* m, int q, int states, float (&v)[NS]) {
    if (states == kQuad * NS) {
        __builtin_memcpy(v, m + q * NS, sizeof v);
    } else {
#pragma unroll
        for (int s = 0; s < NS; ++s) v[s] = m[min(q * NS + s, states - 1)];
#pragma unroll
        for (int s = 0; s < NS; ++s) v[s] = q * NS + s < states ? v[s] : 0.0f;
    }
}

// B or C of rows [t, t + n), n <= kScanTile, as fp32; states past N and rows past n are zero
template <typename T, int NS>
__device__ __forceinline__ void stage(float* lds, const T* m, int64_t ld, int group_offset, int states, int t, int n) {
    constexpr int NP = kQuad * NS;
    for (int i = threadIdx.x; i < kScanTile * NP; i += kScanWaves * kWave) {
        const int r = i / NP, s = i % NP;
        lds[i] = r < n && s < states ? (float)m[(int64_t)(t + r) * ld + group_offset + s] : 0.0f;
    }
}

// own + h 2^x for the x of a whole chunk or more, given half of it.  Where the
// decay grows (A and the step of the same sign) 2^x alone may pass fp32's range
// while the sum, as row by row, does not: up to 2^254, which takes every h that
// is no subnormal past that range, the root of 2^x holds it.  Beyond, the root
// is the largest number, so that a state of zero stays zero.  (A NaN that
// fminf drops came from a step or an A, and so is in own too.)
constexpr float kLargest = 0x1.fffffep127f;
__device__ __forceinline__ float carry_on(float own, float h, float half) {
    const float root = fminf(__builtin_amdgcn_exp2f(half), kLargest);
    return fmaf(h * root, root, own);
}

// What the chunks leave to one another, for one channel and state: walks the
// `chunks` values m[i * each + e] from the first to the last (or the other way)
// and turns each into own + exp(A S) * (the one before), where one sequence
// passes through the chunk, and leaves it otherwise (read or not).  The walk is
// cut into gridDim.y pieces; each begins at the first chunk of its own that
// takes nothing from the one before, and goes on to the next piece's beginning.
// It waits for memory, not for arithmetic: kCarryBatch chunks are loaded while
// the ones before them are worked on.  Threads that are not live take part in
// the search for the beginning and write nothing: what they read may be written
// by the thread whose value it is.
constexpr int kCarryBatch = 16;

__device__ __forceinline__ void carry_walk(float* m, const ScanArgs& a, int64_t each, int64_t e, int c, float a2, bool live, bool forward) {
    const int n = a.chunks, piece = blockIdx.y, pieces = gridDim.y;
    auto place = [&](int i) { return forward ? i : n - 1 - i; };
    const int from = (int)((int64_t)n * piece / pieces), to = (int)((int64_t)n * (piece + 1) / pieces);
    int begin = to;
    for (int i = from; i < to; i += kWave) {
        const int k = i + (int)(threadIdx.x % kWave);
        const uint64_t fresh = __ballot(k < to && !(a.flags[place(min(k, to - 1))] & kThrough));
        if (fresh) {
            begin = i + __builtin_ctzll(fresh);
            break;
        }
    }
    if (begin >= to || !live) return;
    constexpr int U = kCarryBatch;
    float own[U], span[U], next_own[U], next_span[U];
    uint32_t next_f[U];
    auto load = [&](int i0) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t at = place(min(i0 + u, n - 1));
            next_f[u] = (uint32_t)a.flags[at];
            next_own[u] = m[at * each + e];      // of any value where nothing reads it
            next_span[u] = a.span[at * a.channels + c];
        }
    };
    float v = 0.0f;
    load(begin);
    for (int i0 = begin; i0 < n; i0 += U) {
        int f[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            f[u] = uniform((int)next_f[u]);
            own[u] = next_own[u];
            span[u] = next_span[u];
        }
        if (i0 + U < n) load(i0 + U);
        // the batch's chunks of this walk: up to the end, or to where the next piece begins
        int count = min(U, n - i0);
#pragma unroll
        for (int u = U - 1; u >= 0; --u)
            if (i0 + u >= to && !(f[u] & kThrough)) count = min(count, u);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            v = f[u] & kThrough ? carry_on(own[u], v, 0.5f * a2 * span[u]) : own[u];
            own[u] = v;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            arrive(next_f[u]);
            arrive(next_own[u]);
            arrive(next_span[u]);
        }
        if (count == U) {
#pragma unroll
            for (int u = 0; u < U; ++u) m[place(i0 + u) * each + e] = own[u];
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (u < count) m[place(i0 + u) * each + e] = own[u];
            return;
        }
    }
}

// Pieces of that walk: short ones find their beginning soon, where sequences end often
inline unsigned carry_pieces(int64_t chunks) { return (unsigned)(chunks < 16 ? 1 : chunks / 8 < 32 ? chunks / 8 : 32); }

// What comes to a chunk from its neighbour `from` and the ones that lie `step`
// behind it, m[k] decayed over the chunks between.  After a carry kernel the
// neighbour holds all of it.  Without one (look) the values are the chunks'
// own, and this goes on as far as the sequence does; the loads of U chunks do
// not wait for one another.
template <int NS, int CH>
__device__ __forceinline__ void carried(const float* m, const ScanArgs& a, const Lane<CH>& l, const float (&a2)[CH][NS], int from, int step, bool look, float (&h)[CH][NS]) {
    constexpr int NP = kQuad * NS, U = NS * CH <= 4 ? 8 : NS * CH <= 8 ? 4 : NS * CH <= 16 ? 2 : 1;
    auto own = [&](int k, float (&v)[CH][NS]) {
#pragma unroll
        for (int i = 0; i < CH; ++i) __builtin_memcpy(v[i], m + ((int64_t)k * a.channels + (l.c + i)) * NP + l.q * NS, sizeof v[i]);
    };
    own(from, h);
    if (!look) return;
    float span[CH] = {};
    for (int k = from;; k += U * step) {
        int f[U];
        float d[U][CH], v[U][CH][NS];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int between = min(max(k + u * step, 0), a.chunks - 1);
            f[u] = a.flags[between];
#pragma unroll
            for (int i = 0; i < CH; ++i) d[u][i] = a.span[(int64_t)between * a.channels + (l.c + i)];
            own(min(max(k + (u + 1) * step, 0), a.chunks - 1), v[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int next = k + (u + 1) * step;
            if (!(uniform(f[u]) & kThrough) || next < 0 || next >= a.chunks) return;
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                span[i] += 0.5f * d[u][i];
#pragma unroll
                for (int s = 0; s < NS; ++s) h[i][s] = carry_on(h[i][s], v[u][i][s], a2[i][s] * span[i]);
            }
        }
    }
}

// Whether chunks look for themselves, which saves a launch: where sequences are
// up to `depth` chunks long on average and ragged ones four times that at most.
// The host does not know the lengths of ragged ones, and the rule is a bet on
// even ones: 17 sequences of 8003 x 500 x 16 take 48 us so and 54 with the carry
// kernel, of 3001 x 777 x 24 43 and 51, of 4001 x 1000 x 64 132 and 148; one
// sequence beside three short ones 73 and 63, 68 and 54, 161 and 139.
inline bool look_back(int64_t chunks, int64_t sequences, bool ragged, int64_t depth) {
    return chunks <= depth * sequences && (!ragged || chunks <= 4 * depth);
}

// Whether a lane holds one channel instead of a pair: a single channel has no
// neighbour to read, and few channels and rows fill the chip better with waves
// of half the work; pairs share B, C and their loads.  Of 16 states, one
// sequence, singly and in pairs: 2500 x 1000 42 and 48 us, gradients 106 and 109;
// 3001 x 1111 50 and 55, 131 and 132; 2048 x 2048 49 and 52, 135 and 123; 8192 x
// 1024 89 and 91, 236 and 226; 16384 x 2048 307 and 275.  The gradients change
// sides near 2^22 channels and rows, the scan alone only behind 2^23.
inline bool narrow(const im2win_scan_desc* d) {
    return d->channels == 1 || d->channels * d->tokens < (int64_t(1) << 22);
}

// Compiled shapes: f(NS, CH) for N states; from 32 states a lane's registers
// hold one channel's
template <typename F>
void with_states(int64_t n, bool one, F f) {
    using std::integral_constant;
    using One = integral_constant<int, 1>;
    using Two = integral_constant<int, 2>;
    auto shape = [&](auto ns) {
        if (one) f(ns, One{});
        else f(ns, Two{});
    };
    if (n <= 8) shape(integral_constant<int, 2>{});
    else if (n <= 16) shape(integral_constant<int, 4>{});
    else if (n <= 24) shape(integral_constant<int, 6>{});
    else if (n <= 32) f(integral_constant<int, 8>{}, One{});
    else if (n <= 64) f(integral_constant<int, 16>{}, One{});
    else f(integral_constant<int, 32>{}, One{});
}

// Checks and geometry that the entry points share (seq_scan.hip)
int check_scan(const im2win_scan_desc* d, bool sequences, const int32_t* starts, bool have_starts);
int check_scan_inputs(const im2win_scan_desc* d, const void* x, const void* dt, const float* A, const void* B,
                      const void* C, const float* D, const void* z, const float* dt_bias);
ScanArgs scan_args(const im2win_scan_desc* d, const void* x, const void* dt, const float* A, const void* B,
                   const void* C, const float* D, const void* z, const float* dt_bias, int ch);

}  // namespace im2win
