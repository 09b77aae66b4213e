// What the kernels of window attention share: matrix fragments, tiles of keys,
// values, queries or gradients in LDS, tiles of packed sequences.
//
// All products are 32 x 32 blocks of the matrix cores with the scores held
// transposed: S^T = K Q^T has a query in each column, that is in each lane (and
// its partner 32 lanes on), so the statistics of a row of the softmax are the
// lane's own, and the weights leave the accumulators in the order in which the
// next product reads them as its right operand: an accumulator's registers
// 8 s .. 8 s + 7 hold the rows 16 s + 8 (j / 4) + 4 (lane / 32) + j % 4, and
// the left operand is read from LDS in that order of its inner index.
#pragma once

#include "seq_common.h"

#include <algorithm>
#include <type_traits>

namespace im2win {

constexpr int kAttnThreads = 256;      // 4 waves
constexpr int kCols = 32;              // columns (a query of a head each) of a wave
constexpr int kGroupCols = 128;        // of a workgroup
constexpr int kMaxSinks = 32;
constexpr float kLog2e = 1.44269504088896f;
constexpr float kLn2 = 0.693147180559945f;

using f32x16 = float __attribute__((ext_vector_type(16)));
using bf16x8 = __bf16 __attribute__((ext_vector_type(8)));
using s16x4 = short __attribute__((ext_vector_type(4)));

// Eight elements of a lane: 16 of the inner index in a wave's two halves.
template <typename T> struct Frag;
template <> struct Frag<bf16> {
    bf16x8 v;
    __device__ __forceinline__ void load(const void* p) { __builtin_memcpy(&v, p, 16); }
    __device__ __forceinline__ void zero() { v = bf16x8{}; }
    __device__ __forceinline__ float get(int i) const { return (float)v[i]; }
    __device__ __forceinline__ void set(int i, float x) { v[i] = (bf16)x; }
};
template <> struct Frag<float> {
    float v[8];
    __device__ __forceinline__ void load(const void* p) { __builtin_memcpy(v, p, 32); }
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0.0f;
    }
    __device__ __forceinline__ float get(int i) const { return v[i]; }
    __device__ __forceinline__ void set(int i, float x) { v[i] = x; }
};

// acc += A B over the 16 inner values of both halves.  fp32 has no instruction
// of that depth: element j of all lanes is one of depth 2.
__device__ __forceinline__ void mma(f32x16& acc, const Frag<bf16>& a, const Frag<bf16>& b) {
    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.v, b.v, acc, 0, 0, 0);
}
__device__ __forceinline__ void mma(f32x16& acc, const Frag<float>& a, const Frag<float>& b) {
#pragma unroll
    for (int j = 0; j < 8; ++j) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a.v[j], b.v[j], acc, 0, 0, 0);
}

// Sixteen values of an accumulator as a product's right operand.  In bf16 they
// go in two parts, the rounding to bf16 and what it leaves (together off by
// 2^-17): weights and ds of one part would add an error as large as an output's
// own rounding.
template <typename T> struct Parts;
template <> struct Parts<float> {
    Frag<float> high;
    __device__ __forceinline__ Parts(const f32x16& s, int part) {
#pragma unroll
        for (int j = 0; j < 8; ++j) high.v[j] = s[8 * part + j];
    }
};
template <> struct Parts<bf16> {
    Frag<bf16> high, low;
    __device__ __forceinline__ Parts(const f32x16& s, int part) {
        uint32_t h[4], l[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {      // from the pair's word: from its elements, each would be rounded once more
            const float x = s[8 * part + 2 * j], y = s[8 * part + 2 * j + 1];
            h[j] = pair(x, y);
            l[j] = pair(x - __uint_as_float(h[j] << 16), y - __uint_as_float(h[j] & 0xffff0000u));
        }
        __builtin_memcpy(&high, h, 16);
        __builtin_memcpy(&low, l, 16);
    }

protected:
    __device__ __forceinline__ Parts() {}
    static __device__ __forceinline__ uint32_t pair(float x, float y) {
        const __bf16 __attribute__((ext_vector_type(2))) v = {(bf16)x, (bf16)y};
        uint32_t u;
        __builtin_memcpy(&u, &v, 4);
        arrive(u);
        return u;
    }
};

// Weights, which are not negative: the first part is cut off, not rounded, and
// 2^-24 of it is added to the second, which then is zero with the weight alone: an
// infinity times both is one (together off by 2^-16).
template <typename T> struct Weights : Parts<T> {
    using Parts<T>::Parts;
};
template <> struct Weights<bf16> : Parts<bf16> {
    __device__ __forceinline__ Weights(const f32x16& s, int part) {
        uint32_t h[4], l[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t x = __float_as_uint(s[8 * part + 2 * j]), y = __float_as_uint(s[8 * part + 2 * j + 1]);
            const uint32_t xh = x & 0xffff0000u, yh = y & 0xffff0000u;
            h[j] = xh >> 16 | yh;
            l[j] = pair(fmaf(__uint_as_float(xh), 0x1p-24f - 1.0f, __uint_as_float(x)), fmaf(__uint_as_float(yh), 0x1p-24f - 1.0f, __uint_as_float(y)));
        }
        __builtin_memcpy(&high, h, 16);
        __builtin_memcpy(&low, l, 16);
    }
};
template <typename T>
__device__ __forceinline__ void mma(f32x16& acc, const Frag<T>& a, const Parts<T>& b) {
    mma(acc, a, b.high);
    if constexpr (sizeof(T) == 2) mma(acc, a, b.low);
}

// Row of accumulator register i
__device__ __forceinline__ int acc_row(int i, int half) { return 8 * (i / 4) + 4 * half + i % 4; }

// ---------------------------------------------------------------------------
// A tile of R rows of DP elements in LDS, in 16-byte chunks whose place among
// eight (four, where the row's chunks are no multiple of eight) is changed by
// the row's number: eight neighbouring rows then lie in different banks where a
// wave reads one chunk of each (scores), and four neighbouring rows where it
// reads two chunks of each (transposed).  A chunk's number splits into a part
// of the lane's and a constant, so an address is the lane's base, one exclusive
// or, and an immediate.
// ---------------------------------------------------------------------------
template <typename T, int DP, int R>
struct Tile {
    static constexpr int kElems = 16 / sizeof(T);
    static constexpr int kChunks = DP / kElems;             // of a row
    static constexpr int kRow = DP * (int)sizeof(T);        // bytes
    static constexpr int kBytes = R * kRow;
    static constexpr int kMask = kChunks % 8 == 0 ? 7 : 3;
    static_assert(kChunks % 4 == 0, "whole groups of chunks");

    static __device__ __forceinline__ int turn(int row) {
        if constexpr (kMask == 7) return (row & 3) << 1 | (row >> 2 & 1);
        else return (row >> 1 & 1) << 1 | (row >> 2 & 1);
    }
    static __device__ __forceinline__ int at(int row, int chunk) { return row * kRow + (chunk ^ turn(row)) * 16; }

    // The left operand for products over the row's elements: row lane % 32 of
    // block `block`, elements 16 s + 8 (lane / 32) ..
    static __device__ __forceinline__ int row_base(int lane) {
        const int row = lane % 32, half = lane / 32;
        return row * kRow + (turn(row) ^ (sizeof(T) == 2 ? half : 2 * half)) * 16;
    }
    static __device__ __forceinline__ Frag<T> row_frag(const char* lds, int base, int block, int s) {
        Frag<T> f;
        if constexpr (sizeof(T) == 2) {
            f.load(lds + (base ^ (2 * s & kMask) * 16) + (2 * s & ~kMask) * 16 + block * 32 * kRow);
        } else {
            __builtin_memcpy(f.v, lds + (base ^ (4 * s & kMask) * 16) + (4 * s & ~kMask) * 16 + block * 32 * kRow, 16);
            __builtin_memcpy(f.v + 4, lds + (base ^ ((4 * s + 1) & kMask) * 16) + (4 * s & ~kMask) * 16 + block * 32 * kRow, 16);
        }
        return f;
    }
    // The left operand for products over rows: element 32 dt + lane % 32 of the
    // rows 16 s + 8 (j / 4) + 4 (lane / 32) + j % 4.  In bf16 the LDS turns blocks
    // of four rows by 16 elements for 16 lanes: lane l of them names row l / 4,
    // elements 4 (l % 4) .., and receives element l of the four rows.
    static __device__ __forceinline__ int col_base(int lane) {
        const int half = lane / 32;
        if constexpr (sizeof(T) == 2) {
            const int l = lane % 16, row = 4 * half + l / 4;
            return row * kRow + (turn(row) ^ (lane / 16 % 2 * 2 + l % 4 / 2)) * 16 + l % 2 * 8;
        } else {
            return 4 * half * kRow + (turn(4 * half) ^ (lane % 32 / 4)) * 16 + lane % 4 * 4;
        }
    }
    static __device__ __forceinline__ Frag<T> col_frag(const char* lds, int base, int dt, int s) {
        Frag<T> f;
        if constexpr (sizeof(T) == 2) {
            const char* p = lds + (base ^ (4 * dt & kMask) * 16) + (4 * dt & ~kMask) * 16 + 16 * s * kRow;
            union {
                s16x4 h[2];
                bf16x8 v;
            } u;
            u.h[0] = turned(p);
            u.h[1] = turned(p + 8 * kRow);
            f.v = u.v;
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)      // turn(4 half + j % 4) = turn(4 half) ^ 2 (j % 4)
                f.v[j] = *reinterpret_cast<const float*>(lds + (base ^ (j % 4) * 32) + 8 * dt * 16 + (16 * s + 8 * (j / 4) + j % 4) * kRow);
        }
        return f;
    }

private:
    static __device__ __forceinline__ s16x4 turned(const char* p) {
        typedef __attribute__((address_space(3))) s16x4 lds_vec;
        return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_vec*)(p));
    }
};

// 16 bytes in flight
struct Chunk {
    uint32_t __attribute__((ext_vector_type(4))) u;
    __device__ __forceinline__ void zero() { u = 0; }
    __device__ __forceinline__ void load(const void* p) { __builtin_memcpy(&u, p, 16); }
    __device__ __forceinline__ void store(void* p) const { __builtin_memcpy(p, &u, 16); }
};

// ---------------------------------------------------------------------------
// A tile's way from rows in memory to LDS: copied by the memory pipeline
// itself, 16 bytes a lane, without registers.  A lane's place in LDS is fixed
// (64 lanes side by side), so it fetches the chunk that belongs there.
// ---------------------------------------------------------------------------
constexpr int64_t kMaxAttnStride = int64_t(1) << 24;      // a tile's 64 rows of bf16 or 32 of fp32 within 32 bits of bytes

// Tiles are copied this many ahead of the one that is worked on: two where one
// workgroup a CU has LDS for three pairs of them, since no other covers the
// copies' way then (2503 tokens fp32: 209 -> 189 us, as they first ran); with more
// workgroups one (two took 238 us where one took 195, by the registers that they cost).
template <int BYTES, int WAVES> constexpr int kAheadTiles = WAVES == 1 && 3 * 2 * BYTES <= 156 * 1024 ? 2 : 1;

// The wave's copies but for the newest N have arrived, and then everyone's.
// N may only count copies that each wave has issued whatever its lanes hold.
template <int N>
__device__ __forceinline__ void arrived(bool all_but_newest) {
    static_assert(N < 64, "the counter's range");
    if (all_but_newest) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
}

template <typename T, int DP, int R>
struct Feed {
    using Lds = Tile<T, DP, R>;
    static constexpr int kPasses = R * Lds::kChunks / kAttnThreads;
    static_assert(R * Lds::kChunks % kAttnThreads == 0, "whole passes");
    // where a pass is a multiple of eight rows, a lane's chunk is the same in all of them
    static constexpr bool kSame = kAttnThreads % (8 * Lds::kChunks) == 0;
    static constexpr int kPassRows = kAttnThreads / Lds::kChunks;

    static __device__ __forceinline__ int row(int i) { return ((int)threadIdx.x + i * kAttnThreads) / Lds::kChunks; }
    static __device__ __forceinline__ int chunk(int i) { return ((int)threadIdx.x + i * kAttnThreads) % Lds::kChunks ^ Lds::turn(row(i)); }

    uint32_t offset[kSame ? 1 : kPasses], stride;
    __device__ __forceinline__ explicit Feed(int64_t elements) {
        stride = (uint32_t)elements * (uint32_t)sizeof(T);
#pragma unroll
        for (int i = 0; i < (kSame ? 1 : kPasses); ++i) offset[i] = (uint32_t)row(i) * stride + (uint32_t)chunk(i) * 16;
    }
    static __device__ __forceinline__ void copy(const void* from, char* lds, int i) {
        typedef __attribute__((address_space(3))) void lds_void;
        char* to = lds + (uniform((int)threadIdx.x / kWave) * kWave + i * kAttnThreads) * 16;
        __builtin_amdgcn_global_load_lds(from, (lds_void*)(to), 16, 0, 0);
    }
    // The tile's first row is at p and `valid` rows exist (1 at least): behind
    // them the last one is repeated.  Channels behind dim are left alone.
    __device__ __forceinline__ void issue(char* lds, const char* p, int valid, int dim) const {
        if (valid >= R && dim == DP) {
#pragma unroll
            for (int i = 0; i < kPasses; ++i) copy(p + (kSame ? (int64_t)(i * kPassRows) * stride : 0) + offset[kSame ? 0 : i], lds, i);
        } else {
#pragma unroll
            for (int i = 0; i < kPasses; ++i) {
                const int r = row(i) < valid ? row(i) : valid - 1;
                if (chunk(i) * Lds::kElems < dim) copy(p + (int64_t)r * stride + chunk(i) * 16, lds, i);
            }
        }
    }
};

// Zeroes LDS whose channels behind dim no copy writes
__device__ __forceinline__ void clear(char* lds, int bytes) {
    Chunk z;
    z.zero();
    for (int i = threadIdx.x * 16; i < bytes; i += kAttnThreads * 16) z.store(lds + i);
    __syncthreads();
}

// Writes four neighbouring channels
__device__ __forceinline__ void put4(float* p, float a, float b, float c, float d) {
    const float v[4] = {a, b, c, d};
    __builtin_memcpy(p, v, 16);
}
__device__ __forceinline__ void put4(bf16* p, float a, float b, float c, float d) {
    const uint32_t v[2] = {pack_bf16(a, b), pack_bf16(c, d)};
    __builtin_memcpy(p, v, 8);
}

// The sum, or the largest, of both halves' values
__device__ __forceinline__ float half_sum(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float half_max(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// Whether a chunk holds an infinity or a NaN (an exponent of ones carries over when one is added)
template <typename T>
__device__ __forceinline__ bool nonfinite(const Chunk& c) {
    uint32_t any = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        any |= sizeof(T) == 4 ? (c.u[i] & 0x7f800000u) + 0x00800000u : (c.u[i] & 0x7f807f80u) + 0x00800080u;
    return any & (sizeof(T) == 4 ? 0x80000000u : 0x80008000u);
}

// Zeroes the infinities and NaN among a chunk's elements
template <typename T>
__device__ __forceinline__ void drop_nonfinite(Chunk& c) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) {
            if ((c.u[i] & 0x7f800000u) == 0x7f800000u) c.u[i] = 0;
        } else {
            if ((c.u[i] & 0x7f80u) == 0x7f80u) c.u[i] &= 0xffff0000u;
            if ((c.u[i] & 0x7f800000u) == 0x7f800000u) c.u[i] &= 0x0000ffffu;
        }
    }
}

template <typename T>
__device__ __forceinline__ bool finite(T x) {
    return (__float_as_uint((float)x) & 0x7f800000u) != 0x7f800000u;
}
// Whether one of a lane's sums is not finite
template <int N>
__device__ __forceinline__ bool nonfinite(const f32x16 (&o)[N]) {
    float z = 0.0f;      // zero times a finite value is zero
#pragma unroll
    for (int t = 0; t < N; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) z = fmaf(o[t][i], 0.0f, z);
    return !(z == 0.0f);
}

// ---------------------------------------------------------------------------
// Tiles of `rows` rows of the sequences.  The host does not know the
// sequences' lengths, so sequence b owns the places first(b) / rows + b and
// up to the next one's: as many as its rows need, or one more, and there are
// tokens / rows + sequences places in all.
// ---------------------------------------------------------------------------
struct SeqTile {
    int b, first, len, row;      // the sequence, its first row and length, the tile's first row in it (len and more: nothing to do)
};

// The tile at a place, where seq_starts is given and sequence b's places begin at
// first_place(b), which does not decrease.
template <typename F>
__device__ __forceinline__ SeqTile find_tile(const SeqMap& seq, int place, int rows, F first_place) {
    SeqTile t;
    const int lane = threadIdx.x % kWave;
    int lo = 0, n = seq.count;
    while (n > kWave - 1) {
        const int step = (n + kWave - 2) / (kWave - 1), i = lo + lane * step;
        const uint64_t in = __ballot(i < seq.count && first_place(i < seq.count ? i : 0) <= place) | 1;
        lo += (63 - __builtin_clzll(in)) * step;
        n = seq.count - lo < step ? seq.count - lo : step;
    }
    const int i = lo + lane;
    const uint64_t in = __ballot(lane < n && first_place(i < seq.count ? i : 0) <= place) | 1;
    t.b = uniform(lo + 63 - __builtin_clzll(in));
    t.first = seq.first(t.b);
    t.len = seq.first(t.b + 1) - t.first;
    const int64_t row = (int64_t)(place - uniform(first_place(t.b))) * rows;
    t.row = row < 0 || row > t.len ? (t.len > 0 ? t.len : 0) : (int)row;      // (below zero only where seq_starts decreases)
    return t;
}
__device__ __forceinline__ SeqTile seq_tile(const SeqMap& seq, int place, int rows) {
    if (seq.starts) return find_tile(seq, place, rows, [&](int b) { return seq.clamped(b) / rows + b; });
    SeqTile t;
    const int per = (seq.len + rows - 1) / rows;
    t.b = uniform(place / per);
    t.first = t.b * seq.len;
    t.len = seq.len;
    t.row = (place - t.b * per) * rows;
    return t;
}
inline int64_t seq_places(int64_t tokens, int64_t sequences, const int32_t* starts, int64_t rows) {
    if (!starts) {
        const int64_t len = tokens / sequences;
        return sequences * ((len + rows - 1) / rows);
    }
    return tokens / rows + sequences;
}

// Workgroups go to the eight dies in turn; neighbouring places, which read the
// same keys, go to the same one.  `n` work items, launched as a multiple of 8.
__device__ __forceinline__ int64_t die_order(int64_t id, int64_t n) {
    const int64_t per = (n + 7) / 8;
    return id % 8 * per + id / 8;
}

// f(head size the kernels are compiled for)
template <typename F>
void with_head(int64_t dim, F f) {
    using std::integral_constant;
    if (dim <= 32) f(integral_constant<int, 32>{});
    else if (dim <= 64) f(integral_constant<int, 64>{});
    else if (dim <= 96) f(integral_constant<int, 96>{});
    else if (dim <= 128) f(integral_constant<int, 128>{});
    else if (dim <= 192) f(integral_constant<int, 192>{});
    else f(integral_constant<int, 256>{});
}

// Heads that share a wave's columns: all of a group's, or the largest divisor
// of their number that leaves a wave whole ones.
inline int heads_packed(int64_t q_heads, int64_t kv_heads) {
    const int64_t group = q_heads / kv_heads;
    int best = 1;
    for (int p = 1; p <= kCols && p <= group; ++p)
        if (group % p == 0) best = p;
    return best;
}

inline int check_attention(const im2win_window_desc* d) {
    if (!d) return fail(IM2WIN_ENULL, "descriptor is NULL");
    int rc = check_rows(d->tokens, 1, d->dtype);
    if (rc) return rc;
    // positions, with up to 2^30 tokens before the call and a tile behind the last, stay in 32 bits
    if (d->tokens > (int64_t(1) << 29)) return fail(IM2WIN_EOVERFLOW, "at most 2^29 tokens (got %lld)", (long long)d->tokens);
    if (d->kv_heads < 1 || d->q_heads < 1 || d->q_heads > 65536 || d->q_heads % d->kv_heads)
        return fail(IM2WIN_EINVAL, "q_heads must be 1 to 65536 and a multiple of kv_heads (got %lld, %lld)", (long long)d->q_heads, (long long)d->kv_heads);
    if (d->head_dim < 8 || d->head_dim > 256 || d->head_dim % 8)
        return fail(IM2WIN_EINVAL, "head_dim must be a multiple of 8 up to 256 (got %lld)", (long long)d->head_dim);
    if (d->window < 1 || d->sinks < 0 || d->sinks > kMaxSinks)
        return fail(IM2WIN_EINVAL, "window must be >= 1 and sinks 0 to %d (got %lld, %lld)", kMaxSinks, (long long)d->window, (long long)d->sinks);
    if (d->window > (int64_t(1) << 30)) return fail(IM2WIN_EOVERFLOW, "at most a window of 2^30 (got %lld)", (long long)d->window);
    if (!(d->scale > 0.0f) || d->scale > 1e30f) return fail(IM2WIN_EINVAL, "scale must be positive (got %g)", (double)d->scale);
    if ((rc = check_ld(d->ld_q, d->q_heads * d->head_dim, "ld_q")) || (rc = check_ld(d->ld_k, d->kv_heads * d->head_dim, "ld_k")) ||
        (rc = check_ld(d->ld_v, d->kv_heads * d->head_dim, "ld_v")))
        return rc;
    if (std::max({d->ld_q, d->ld_k, d->ld_v}) >= kMaxAttnStride)
        return fail(IM2WIN_EOVERFLOW, "row strides stay below 2^24 (got %lld, %lld, %lld)", (long long)d->ld_q, (long long)d->ld_k, (long long)d->ld_v);
    return IM2WIN_OK;
}

}  // namespace im2win
