// What the sequence operators (include/im2win_seq.h) share: element types,
// rows of packed sequences, lane exchanges.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "error.h"
#include "im2win_seq.h"

namespace im2win {

using bf16 = __bf16;   // conversions from float round to nearest even

constexpr int kWave = 64;
// Rows are counted in 32-bit integers with room for a tile past the end.
constexpr int64_t kMaxTokens = (int64_t(1) << 31) - (int64_t(1) << 20);
constexpr int64_t kMaxChannels = int64_t(1) << 20;

// ---------------------------------------------------------------------------
// Sequences in the rows.  Every bound a kernel uses comes from first(), which
// lies in [0, tokens] whatever seq_starts holds.
// ---------------------------------------------------------------------------
struct SeqMap {
    const int32_t* starts;   // NULL: sequences of `len` rows each
    int count;
    int len;
    int tokens;

    __device__ int first(int b) const {
        if (!starts) return b * len;   // b <= count, count * len == tokens
        const int s = starts[b];
        return s < 0 ? 0 : s > tokens ? tokens : s;
    }
    // The sequence that holds row t, for first(0) <= t < first(count).
    __device__ int find(int t) const {
        if (!starts) return t / len;
        int lo = 0, hi = count;        // starts[lo] <= t < starts[hi]
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (first(mid) <= t) lo = mid; else hi = mid;
        }
        return lo;
    }
};

inline SeqMap make_seq_map(int64_t tokens, int64_t sequences, const int32_t* starts) {
    SeqMap m;
    m.starts = starts;
    m.count = (int)sequences;
    m.len = (int)(tokens / sequences);
    m.tokens = (int)tokens;
    return m;
}

// ---------------------------------------------------------------------------
// V consecutive elements, as fp32.  V > 1 means 16 bytes at a 16-byte aligned
// address (4 floats, 8 bfloat16).
// ---------------------------------------------------------------------------
template <typename T> constexpr int kVec = 16 / sizeof(T);

template <int V>
__device__ __forceinline__ void load_vec(const float* p, float (&v)[V]) {
    if constexpr (V == 1) {
        v[0] = p[0];
    } else {
        static_assert(V == 4, "16 bytes");
        const float4 r = *reinterpret_cast<const float4*>(p);
        v[0] = r.x; v[1] = r.y; v[2] = r.z; v[3] = r.w;
    }
}

template <int V>
__device__ __forceinline__ void load_vec(const bf16* p, float (&v)[V]) {
    if constexpr (V == 1) {
        v[0] = (float)p[0];
    } else {
        static_assert(V == 8, "16 bytes");
        const uint4 r = *reinterpret_cast<const uint4*>(p);
        const uint32_t u[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(u[i] << 16);
            v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
        }
    }
}

template <int V>
__device__ __forceinline__ void store_vec(float* p, const float (&v)[V]) {
    if constexpr (V == 1) {
        p[0] = v[0];
    } else {
        static_assert(V == 4, "16 bytes");
        *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    }
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    return (uint32_t)__builtin_bit_cast(uint16_t, (bf16)lo) |
           (uint32_t)__builtin_bit_cast(uint16_t, (bf16)hi) << 16;
}

template <int V>
__device__ __forceinline__ void store_vec(bf16* p, const float (&v)[V]) {
    if constexpr (V == 1) {
        p[0] = (bf16)v[0];
    } else {
        static_assert(V == 8, "16 bytes");
        *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]),
                                                  pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
    }
}

// fp32 arrays of a multiple of four, on 16-byte boundaries when V > 1
template <int V>
__device__ __forceinline__ void store_f32(float* p, const float (&v)[V]) {
    if constexpr (V % 4 == 0) {
#pragma unroll
        for (int i = 0; i < V; i += 4)
            *reinterpret_cast<float4*>(p + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) p[i] = v[i];
    }
}

// 1 / (1 + exp(-v)): the exponential and the reciprocal are the hardware's
// (about one unit in the last place each); far negative v gives 0.
__device__ __forceinline__ float sigmoid(float v) {
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504088896f * v));
}

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
inline bool aligned_to(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// A pointer an entry point needs (or may have): not NULL, aligned to its element.
inline int need_ptr(const void* p, size_t align, const char* name) {
    if (!p) return fail(IM2WIN_ENULL, "%s is NULL", name);
    if (!aligned_to(p, align)) return fail(IM2WIN_EALIGN, "%s (%p) is not %zu-byte aligned", name, p, align);
    return IM2WIN_OK;
}
inline int may_ptr(const void* p, size_t align, const char* name) {
    return p ? need_ptr(p, align, name) : IM2WIN_OK;
}

// Row counts, sequences and element type that every descriptor shares.
inline int check_rows(int64_t tokens, int64_t channels, int32_t dtype) {
    if (tokens < 0 || channels < 1)
        return fail(IM2WIN_EINVAL, "tokens must be >= 0 and channels >= 1 (got %lld, %lld)",
                    (long long)tokens, (long long)channels);
    if (dtype != IM2WIN_F32 && dtype != IM2WIN_BF16) return fail(IM2WIN_EINVAL, "unknown dtype %d", (int)dtype);
    if (tokens > kMaxTokens || channels > kMaxChannels)
        return fail(IM2WIN_EOVERFLOW, "at most %lld tokens of %lld channels (got %lld, %lld)", (long long)kMaxTokens,
                    (long long)kMaxChannels, (long long)tokens, (long long)channels);
    return IM2WIN_OK;
}

inline int check_sequences(int64_t tokens, int64_t sequences, const int32_t* starts, bool have_starts) {
    if (sequences < 1) return fail(IM2WIN_EINVAL, "sequences must be >= 1 (got %lld)", (long long)sequences);
    if (sequences > kMaxTokens) return fail(IM2WIN_EOVERFLOW, "too many sequences (%lld)", (long long)sequences);
    if (have_starts && !starts && tokens % sequences)
        return fail(IM2WIN_EINVAL, "%lld tokens are not %lld sequences of the same length (give seq_starts)",
                    (long long)tokens, (long long)sequences);
    return may_ptr(starts, 4, "seq_starts");
}

// Row strides stay below 2^31 elements, so that a row times its stride, in bytes, fits 64 bits.
inline int check_ld(int64_t ld, int64_t width, const char* name) {
    if (ld < width)
        return fail(IM2WIN_EINVAL, "%s is %lld, less than the row's %lld elements", name, (long long)ld, (long long)width);
    if (ld > (int64_t(1) << 31) - 1) return fail(IM2WIN_EOVERFLOW, "%s (%lld) exceeds 2^31 - 1", name, (long long)ld);
    return IM2WIN_OK;
}

inline int launched(const char* what) {
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(IM2WIN_EHIP, "%s launch failed: %s", what, hipGetErrorString(e));
    return ok();
}

}  // namespace im2win
