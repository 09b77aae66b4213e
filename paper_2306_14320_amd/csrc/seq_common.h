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

// A value that is the same in every lane of the wave, held in a scalar register.
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// Waits for a load whose result is v, here and not where v is used.  Loads and
// stores come back in one order, so a wait for a prefetched value that stands
// behind stores waits for those too: it is put in front of them.
__device__ __forceinline__ void arrive(uint32_t& v) { asm volatile("" : "+v"(v)); }
__device__ __forceinline__ void arrive(float& v) { asm volatile("" : "+v"(v)); }

// ---------------------------------------------------------------------------
// Sequences in the rows.  Every bound a kernel uses comes from first(), which
// lies in [0, tokens] whatever seq_starts holds.  Arguments are wave-uniform.
// ---------------------------------------------------------------------------
struct SeqMap {
    const int32_t* starts;   // NULL: sequences of `len` rows each
    int count;
    int len;
    int tokens;

    __device__ int first(int b) const {
        if (!starts) return b * len;   // b <= count, count * len == tokens
        const int s = uniform(starts[b]);
        return s < 0 ? 0 : s > tokens ? tokens : s;
    }
    // The sequence that holds row t, for first(0) <= t < first(count), and its
    // rows.  The wave's lanes, all of them active, look at 64 starts at a time,
    // so that up to 63 sequences take one load's latency and 4000 two.
    struct Found {
        int b, first, end;
    };
    __device__ Found at(int t) const {
        Found f;
        if (!starts) {
            f.b = uniform(t / len);
            f.first = f.b * len;
            f.end = f.first + len;
            return f;
        }
        const int lane = threadIdx.x % kWave;
        auto look = [&](int i) {
            const int s = starts[i < count ? i : count];
            return s < 0 ? 0 : s > tokens ? tokens : s;
        };
        int lo = 0, n = count;         // one of the sequences [lo, lo + n); starts[lo] <= t
        while (n > kWave - 1) {
            const int step = (n + kWave - 2) / (kWave - 1);
            const uint64_t before = __ballot(look(lo + lane * step) <= t) | 1;
            lo += (63 - __builtin_clzll(before)) * step;
            n = count - lo < step ? count - lo : step;
        }
        const int s = look(lo + lane);
        const int k = 63 - __builtin_clzll(__ballot(lane < n && s <= t) | 1);
        f.b = uniform(lo + k);
        f.first = __builtin_amdgcn_readlane(s, k);
        f.end = __builtin_amdgcn_readlane(s, k + 1);
        return f;
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
// V consecutive elements: one, or 16 bytes of them (4 floats, 8 bfloat16) in
// one access.  Addresses need the alignment of an element only: the hardware
// takes 16 bytes from any address (the norm's gradients of 8191 x 2049 rows
// take 59 us so, and took 203 element by element).
// ---------------------------------------------------------------------------
template <typename T> constexpr int kVec = 16 / sizeof(T);

// V elements as they lie in memory; get() converts, so that a load can stay
// in flight until its value is used.
template <typename T, int V>
struct Bits {
    static_assert(V == kVec<T>, "16 bytes");
    uint32_t u[4];
    __device__ __forceinline__ void load(const T* p) { __builtin_memcpy(u, p, 16); }
    __device__ __forceinline__ void zero() { u[0] = u[1] = u[2] = u[3] = 0; }
    __device__ __forceinline__ void wait() {
#pragma unroll
        for (int i = 0; i < 4; ++i) arrive(u[i]);
    }
    __device__ __forceinline__ float get(int i) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(u[i]);
        else return __uint_as_float(i % 2 ? u[i / 2] & 0xffff0000u : u[i / 2] << 16);
    }
};
template <typename T>
struct Bits<T, 1> {
    T u;
    __device__ __forceinline__ void load(const T* p) { u = *p; }
    __device__ __forceinline__ void zero() { u = (T)0.0f; }
    __device__ __forceinline__ void wait() {}
    __device__ __forceinline__ float get(int) const { return (float)u; }
};

template <int V, typename T>
__device__ __forceinline__ void load_vec(const T* p, float (&v)[V]) {
    Bits<T, V> r;
    r.load(p);
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = r.get(i);
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    return (uint32_t)__builtin_bit_cast(uint16_t, (bf16)lo) |
           (uint32_t)__builtin_bit_cast(uint16_t, (bf16)hi) << 16;
}

template <int V>
__device__ __forceinline__ void store_vec(float* p, const float (&v)[V]) {
    __builtin_memcpy(p, v, V * sizeof(float));
}

template <int V>
__device__ __forceinline__ void store_vec(bf16* p, const float (&v)[V]) {
    if constexpr (V == 1) {
        p[0] = (bf16)v[0];
    } else {
        const uint32_t u[4] = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
        __builtin_memcpy(p, u, 16);
    }
}

// N consecutive values, a multiple of the vector width
template <int N, typename T>
__device__ __forceinline__ void store_run(T* p, const float (&v)[N]) {
    static_assert(N % kVec<T> == 0, "whole vectors");
#pragma unroll
    for (int i = 0; i < N; i += kVec<T>) {
        float w[kVec<T>];
#pragma unroll
        for (int j = 0; j < kVec<T>; ++j) w[j] = v[i + j];
        store_vec<kVec<T>>(p + i, w);
    }
}

// 1 / (1 + exp(-v)): the exponential and the reciprocal are the hardware's
// (about one unit in the last place each); far negative v gives 0.
__device__ __forceinline__ float sigmoid(float v) {
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504088896f * v));
}

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

// Row strides: four rows' bytes fit 32 bits, as the kernels' offsets inside such a group do.
constexpr int64_t kMaxStride = int64_t(1) << 28;

inline int check_ld(int64_t ld, int64_t width, const char* name) {
    if (ld < width)
        return fail(IM2WIN_EINVAL, "%s is %lld, less than the row's %lld elements", name, (long long)ld, (long long)width);
    if (ld > kMaxStride - 1) return fail(IM2WIN_EOVERFLOW, "%s (%lld) reaches 2^28", name, (long long)ld);
    return IM2WIN_OK;
}

// The runtime takes fewer than 2^32 threads a launch (and dimension): checked
// before the first launch of a call, so that a refused call has written nothing.
constexpr int64_t kMaxThreads = (int64_t(1) << 32) - 1;

inline int check_launch(int64_t blocks, int threads, const char* what) {
    if (blocks > kMaxThreads / threads)
        return fail(IM2WIN_EOVERFLOW, "%s: %lld workgroups of %d threads are more than a launch holds (rows, sequences or channels are too many)",
                    what, (long long)blocks, threads);
    return IM2WIN_OK;
}

inline int launched(const char* what) {
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(IM2WIN_EHIP, "%s launch failed: %s", what, hipGetErrorString(e));
    return ok();
}

}  // namespace im2win
