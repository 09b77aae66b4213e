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

// Row of accumulator register i
__device__ __forceinline__ int acc_row(int i, int half) { return 8 * (i / 4) + 4 * half + i % 4; }

// ---------------------------------------------------------------------------
// A tile of R rows of DP elements in LDS, in 16-byte chunks whose place in the
// row is changed by the row's number: eight neighbouring rows then lie in
// different banks where a wave reads one chunk of each (scores), and four
// neighbouring rows where it reads two chunks of each (transposed).
// ---------------------------------------------------------------------------
template <typename T, int DP, int R>
struct Tile {
    static constexpr int kElems = 16 / sizeof(T);
    static constexpr int kChunks = DP / kElems;             // of a row
    static constexpr int kBytes = R * DP * (int)sizeof(T);

    static __device__ __forceinline__ int turn(int row) {
        if constexpr (kChunks % 8 == 0) return (row & 3) << 1 | (row >> 2 & 1);
        else return (row >> 1 & 1) << 1 | (row >> 2 & 1);
    }
    static __device__ __forceinline__ int at(int row, int chunk) { return (row * kChunks + (chunk ^ turn(row))) * 16; }

    // The left operand for products over the row's elements: row `row`, elements 16 s + 8 half ..
    static __device__ __forceinline__ Frag<T> row_frag(const char* lds, int row, int s, int half) {
        Frag<T> f;
        if constexpr (sizeof(T) == 2) {
            f.load(lds + at(row, 2 * s + half));
        } else {
            __builtin_memcpy(f.v, lds + at(row, 4 * s + 2 * half), 16);
            __builtin_memcpy(f.v + 4, lds + at(row, 4 * s + 2 * half + 1), 16);
        }
        return f;
    }
    // The left operand for products over rows: element 32 dt + lane % 32 of the
    // rows 16 s + 8 (j / 4) + 4 half + j % 4.  In bf16 the LDS turns blocks of
    // four rows by 16 elements for 16 lanes: lane l of them names row l / 4,
    // elements 4 (l % 4) .., and receives element l of the four rows.
    static __device__ __forceinline__ Frag<T> col_frag(const char* lds, int dt, int s, int lane) {
        Frag<T> f;
        const int half = lane / 32;
        if constexpr (sizeof(T) == 2) {
            const int l = lane % 16, row = 16 * s + 4 * half + l / 4;
            const int e = 32 * dt + lane / 16 % 2 * 16 + 4 * (l % 4);
            union {
                s16x4 h[2];
                bf16x8 v;
            } u;
            u.h[0] = turned(lds + at(row, e / 8) + e % 8 * 2);
            u.h[1] = turned(lds + at(row + 8, e / 8) + e % 8 * 2);
            f.v = u.v;
        } else {
            const int e = 32 * dt + lane % 32;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int row = 16 * s + 8 * (j / 4) + 4 * half + j % 4;
                f.v[j] = *reinterpret_cast<const float*>(lds + at(row, e / 4) + e % 4 * 4);
            }
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
// A tile's way from rows in memory to LDS, 16 bytes a thread and pass, through
// registers in which the loads stay in flight.  Threads side by side take a
// row's chunks (their number rounded up to a power of two, so that a thread's
// place in its row is the same in every pass and its address one 32-bit offset
// beside a scalar one).
// ---------------------------------------------------------------------------
constexpr int64_t kMaxAttnStride = int64_t(1) << 24;      // 64 rows of bf16 or 32 of fp32 within 32 bits of bytes

template <typename T, int DP, int R>
struct Stage {
    using Lds = Tile<T, DP, R>;
    static constexpr int up(int n) { return n <= 4 ? 4 : n <= 8 ? 8 : n <= 16 ? 16 : n <= 32 ? 32 : 64; }
    static constexpr int kLanes = up(Lds::kChunks), kPassRows = kAttnThreads / kLanes, kPasses = R / kPassRows;
    static_assert(kPasses >= 1 && R % kPassRows == 0, "whole passes");
    Chunk c[kPasses];

    static __device__ __forceinline__ int row() { return (int)threadIdx.x / kLanes; }
    static __device__ __forceinline__ int chunk() { return (int)threadIdx.x % kLanes; }
    static __device__ __forceinline__ bool inside(int dim) { return chunk() * Lds::kElems < dim; }      // the chunk holds channels
    // Bytes from the tile's first row to the thread's first chunk, for rows `stride` bytes apart
    static __device__ __forceinline__ uint32_t offset(uint32_t stride) { return (uint32_t)row() * stride + (uint32_t)chunk() * 16; }

    // `valid` of the tile's rows exist (all where at least R), the first at p; the others, and channels behind dim, are zeros
    __device__ __forceinline__ void fetch(const char* p, uint32_t offset, uint32_t stride, int valid, int dim) {
        if (valid >= R && (Lds::kChunks * Lds::kElems == dim && Lds::kChunks == kLanes)) {
#pragma unroll
            for (int i = 0; i < kPasses; ++i) {
                c[i].load(p + offset);
                p += (int64_t)kPassRows * stride;
            }
        } else {
            const bool in = inside(dim);
#pragma unroll
            for (int i = 0; i < kPasses; ++i) {
                if (in && row() + i * kPassRows < valid) c[i].load(p + offset);
                else c[i].zero();
                p += (int64_t)kPassRows * stride;
            }
        }
    }
    __device__ __forceinline__ void put(char* lds) const {
        if (Lds::kChunks == kLanes || chunk() < Lds::kChunks) {
#pragma unroll
            for (int i = 0; i < kPasses; ++i) c[i].store(lds + Lds::at(row() + i * kPassRows, chunk()));
        }
    }
};

// Zeroes the infinities and NaN among a chunk's elements; whether there were any.
template <typename T>
__device__ __forceinline__ bool drop_nonfinite(Chunk& c) {
    bool any = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) {
            if ((c.u[i] & 0x7f800000u) == 0x7f800000u) c.u[i] = 0, any = true;
        } else {
            if ((c.u[i] & 0x7f80u) == 0x7f80u) c.u[i] &= 0xffff0000u, any = true;
            if ((c.u[i] & 0x7f800000u) == 0x7f800000u) c.u[i] &= 0x0000ffffu, any = true;
        }
    }
    return any;
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

__device__ __forceinline__ SeqTile seq_tile(const SeqMap& seq, int place, int rows) {
    SeqTile t;
    if (!seq.starts) {
        const int per = (seq.len + rows - 1) / rows;
        t.b = uniform(place / per);
        t.first = t.b * seq.len;
        t.len = seq.len;
        t.row = (place - t.b * per) * rows;
        return t;
    }
    const int lane = threadIdx.x % kWave;
    auto first_place = [&](int b) { return seq.clamped(b) / rows + b; };     // strictly increasing
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
    t.row = (place - (t.first / rows + t.b)) * rows;
    if (t.row < 0) t.row = t.len > 0 ? t.len : 0;      // only where seq_starts decreases
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

inline size_t attn_size_of(int32_t dtype) { return dtype == IM2WIN_F32 ? 4 : 2; }

inline int check_attention(const im2win_window_desc* d) {
    if (!d) return fail(IM2WIN_ENULL, "descriptor is NULL");
    int rc = check_rows(d->tokens, 1, d->dtype);
    if (rc) return rc;
    if (d->tokens > (int64_t(1) << 30)) return fail(IM2WIN_EOVERFLOW, "at most 2^30 tokens (got %lld)", (long long)d->tokens);
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
