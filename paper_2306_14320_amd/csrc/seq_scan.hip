// Selective state space scan (im2win_selective_scan, _step,
// include/im2win_seq.h).
//
// The recurrence h_t = a_t h_{t-1} + b_t runs along the rows, so a long
// sequence with few channels would leave most of the chip idle.  The rows are
// cut into chunks, whatever sequences lie in them:
//   1. scan_kernel<SUMMARY>: for each chunk whose last sequence goes on behind
//      it, the state at its end from a zero (or initial) state, and the sum S
//      of the step sizes that a state from before the chunk passes, which is
//      its decay exp(A S);
//   2. scan_carry_kernel: the states behind the chunks, one after the other;
//   3. scan_kernel: each chunk from the state before it, with the outputs.
// Where sequences are few chunks long, step 3 adds up what comes to a chunk
// itself and step 2 does not run (3001 ragged rows of 777 x 24 fp32: 54 us with
// it, 47 without; see look_back).
// With one chunk, or chunks of whole sequences, only step 3 runs.
//
// Bound by issue slots, not memory: a row, channel and state costs the product
// s A, its exponential (two slots), u B, the recurrence and C h, six slots, five
// in step 1, and a row and channel about forty more (step size, gate,
// conversions, sums over the quad).  8192 x 2048 x 16 bf16 takes 147 us; under
// the profiler 62 in step 1, 11 in step 2 and 84 in step 3, with 87% of the
// slots of steps 1 and 3 taken and 1.7 TB/s of traffic.
#include <algorithm>

#include "seq_scan.h"

namespace im2win {
namespace {

// Values of four rows and the lane's channels, one row per lane of the quad
template <typename T, int CH>
struct Rows {
    Raw<T, CH> x, dt, z;
    __device__ __forceinline__ void wait() {
        x.wait();
        dt.wait();
        z.wait();
    }
};
template <typename T, int CH>
struct Places {
    RowPlace<T> x, dt, z;
    __device__ __forceinline__ Places(const ScanArgs& a, const Lane<CH>& l, int row) : x(a.ld_x, l, row), dt(a.ld_dt, l, row), z(a.ld_z, l, row) {}
    template <bool GATE>
    __device__ __forceinline__ void load(const ScanArgs& a, int t, Rows<T, CH>& r) const {
        r.x.load(x.at(a.x, a.ld_x, t));
        r.dt.load(dt.at(a.dt, a.ld_dt, t));
        if constexpr (GATE)
            if (a.z) r.z.load(z.at(a.z, a.ld_z, t));
    }
};

template <typename T, int NS, int CH, bool SUMMARY>
__global__ __launch_bounds__(kScanWaves * kWave) void scan_kernel(ScanArgs a) {
    constexpr int NP = kQuad * NS;
    __shared__ __align__(16) float sb[kScanTile * NP];
    __shared__ __align__(16) float sc[SUMMARY ? 4 : kScanTile * NP];
    const int block = blockIdx.x % a.blocks, chunk = blockIdx.x / a.blocks;
    const int wave = uniform(threadIdx.x / kWave);

    if (chunk >= a.chunks) {
        // workgroups behind the chunks': the final states of sequences without rows
        if constexpr (!SUMMARY) {
            const int64_t each = (int64_t)a.channels * a.states;
            const int extra = (int)gridDim.x - a.blocks * a.chunks;
            for (int b = blockIdx.x - a.blocks * a.chunks; b < a.seq.count; b += extra) {
                if (a.seq.first(b + 1) > a.seq.first(b)) continue;
                for (int64_t i = threadIdx.x; i < each; i += blockDim.x)
                    a.final_state[b * each + i] = a.init ? a.init[b * each + i] : 0.0f;
            }
        }
        return;
    }

    int lo = max(a.seq.first(0), chunk * a.chunk);
    const int hi = min(a.seq.first(a.seq.count), min(chunk * a.chunk, a.seq.tokens - a.chunk) + a.chunk);
    if (lo >= hi) {
        if (SUMMARY && block == 0 && threadIdx.x == 0) a.flags[chunk] = 0;
        return;
    }
    const SeqMap::Found found = a.seq.at(SUMMARY ? hi - 1 : lo);
    const int first = found.first;
    int b = found.b, end = found.end;
    if constexpr (SUMMARY) {
        if (block == 0 && threadIdx.x == 0)
            a.flags[chunk] = end <= hi ? 0 : first < lo ? kGoesOn | kThrough : kGoesOn;
        if (end <= hi) return;
        lo = max(lo, first);
    }

    Lane<CH> l;
    l.init(a, block, wave);
    const int group_offset = block / a.group_blocks * a.states;
    const float* init = a.init;
    float a2[CH][NS], h[CH][NS], bias[CH], skip[CH];
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        bias[i] = a.dt_bias ? a.dt_bias[l.c + i] : 0.0f;
        skip[i] = !SUMMARY && a.D ? a.D[l.c + i] : 0.0f;
        load_states<NS>(a.A + (int64_t)(l.c + i) * a.states, l.q, a.states, a2[i]);
#pragma unroll
        for (int s = 0; s < NS; ++s) a2[i][s] *= kLog2e;
    }
    auto begin = [&]() {     // the state before the first row of sequence b
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            if (init) {
                load_states<NS>(init + ((int64_t)b * a.channels + l.c + i) * a.states, l.q, a.states, h[i]);
            } else {
#pragma unroll
                for (int s = 0; s < NS; ++s) h[i][s] = 0.0f;
            }
        }
    };
    if (lo == first) {
        begin();
    } else if (SUMMARY || chunk == 0) {
#pragma unroll
        for (int i = 0; i < CH; ++i)
#pragma unroll
            for (int s = 0; s < NS; ++s) h[i][s] = 0.0f;
    } else {
        carried<NS, CH>(a.carry, a, l, a2, chunk - 1, -1, a.look != 0, h);
    }

    auto finish = [&]() {     // the state behind the last row of sequence b
        if (SUMMARY || !a.final_state) return;
#pragma unroll
        for (int i = 0; i < CH; ++i)
#pragma unroll
            for (int s = 0; s < NS; ++s) {
                const int n = l.q * NS + s;
                if (l.live[i] && n < a.states)
                    a.final_state[((int64_t)b * a.channels + l.c + i) * a.states + n] = h[i][s];
            }
    };

    float span[CH] = {};
    Places<T, CH> places(a, l, l.q);
    const RowPlace<T> out(a.channels, l, l.q);
    auto load = [&](int t, Rows<T, CH>& r) {
        // the last group may have fewer than four rows: the lanes past them take its last one
        if (t + kQuad > hi) places = Places<T, CH>(a, l, min(l.q, hi - 1 - t));
        places.template load<!SUMMARY>(a, t, r);
    };
    Rows<T, CH> next;
    load(lo, next);
    for (int tile = lo; tile < hi; tile += kScanTile) {
        const int rows = min(kScanTile, hi - tile);
        __syncthreads();
        stage<T, NS>(sb, static_cast<const T*>(a.B), a.ld_b, group_offset, a.states, tile, rows);
        if constexpr (!SUMMARY)
            stage<T, NS>(sc, static_cast<const T*>(a.C), a.ld_c, group_offset, a.states, tile, rows);
        __syncthreads();
        for (int r = 0; r < rows; r += kQuad) {
            const int t = tile + r;
            const Rows<T, CH> now = next;
            if (t + kQuad < hi) load(t + kQuad, next);
            // the first row's B and C are on their way while the steps are computed
            float bm0[NS], cm0[NS];
            lds_row<NS>(sb + r * NP + l.q * NS, bm0);
            if constexpr (!SUMMARY) lds_row<NS>(sc + r * NP + l.q * NS, cm0);
            float step[CH], in[CH], x[CH], sum[CH];
#pragma unroll
            for (int i = 0; i < CH; ++i) step[i] = now.dt.get(i) + bias[i];
            if (a.softplus)
#pragma unroll
                for (int i = 0; i < CH; ++i) step[i] = softplus(step[i]);
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                x[i] = now.x.get(i);
                in[i] = step[i] * x[i];
                if (SUMMARY && t + l.q < hi) span[i] += step[i];
                sum[i] = 0.0f;
            }
            // one row, whose step and input every lane of the quad has: the lane's part of C h
            auto advance_row = [&](int i, float sj, float ij, const float (&bm)[NS], const float (&cm)[NS]) {
                float acc = 0.0f;
#pragma unroll
                for (int s = 0; s < NS; ++s) {
                    h[i][s] = fmaf(__builtin_amdgcn_exp2f(sj * a2[i][s]), h[i][s], ij * bm[s]);
                    if constexpr (!SUMMARY) acc = fmaf(cm[s], h[i][s], acc);
                }
                return acc;
            };
            if (SUMMARY ? t + kQuad <= hi : t < end && t + kQuad <= min(end, hi)) {
                float sums[kQuad][CH];
                auto token = [&](auto j) {
                    constexpr int J = decltype(j)::value;
                    float bm[NS], cm[NS];
                    if constexpr (J > 0) {
                        lds_row<NS>(sb + (r + J) * NP + l.q * NS, bm);
                        if constexpr (!SUMMARY) lds_row<NS>(sc + (r + J) * NP + l.q * NS, cm);
                    } else {
#pragma unroll
                        for (int s = 0; s < NS; ++s) {
                            bm[s] = bm0[s];
                            cm[s] = cm0[s];
                        }
                    }
#pragma unroll
                    for (int i = 0; i < CH; ++i)
                        sums[J][i] = advance_row(i, quad_get<J>(step[i]), quad_get<J>(in[i]), bm, cm);
                };
                using std::integral_constant;
                token(integral_constant<int, 0>{});
                token(integral_constant<int, 1>{});
                token(integral_constant<int, 2>{});
                token(integral_constant<int, 3>{});
                if constexpr (!SUMMARY)
#pragma unroll
                    for (int i = 0; i < CH; ++i) sum[i] = quad_sums(sums[0][i], sums[1][i], sums[2][i], sums[3][i], l.q);
            } else {
                // a group where a sequence begins or ends, or of fewer than four rows
                for (int j = 0; j < kQuad && t + j < hi; ++j) {
                    if (!SUMMARY && t + j >= end) {
                        if (t + j == end) finish();
                        const SeqMap::Found next_seq = a.seq.at(t + j);
                        b = next_seq.b;
                        end = next_seq.end;
                        begin();
                    }
                    float bm[NS], cm[NS];
                    lds_row<NS>(sb + (r + j) * NP + l.q * NS, bm);
                    if constexpr (!SUMMARY) lds_row<NS>(sc + (r + j) * NP + l.q * NS, cm);
#pragma unroll
                    for (int i = 0; i < CH; ++i) {
                        const int from = (int)(threadIdx.x % kWave) / kQuad * kQuad + j;
                        const float part = quad_sum(advance_row(i, __shfl(step[i], from), __shfl(in[i], from), bm, cm));
                        if (l.q == j) sum[i] = part;
                    }
                }
            }
            if constexpr (!SUMMARY) {
#pragma unroll
                for (int i = 0; i < CH; ++i) sum[i] = fmaf(skip[i], x[i], sum[i]);
                if (a.z)
#pragma unroll
                    for (int i = 0; i < CH; ++i) sum[i] *= now.z.get(i) * sigmoid(now.z.get(i));
                next.wait();
                if (t + l.q < hi) store_channels<T, CH>(out.at(a.y, a.channels, t), l.live, sum);
            }
        }
    }
    if (!SUMMARY && end == hi) finish();     // the chunk's last sequence ends with it
    if constexpr (SUMMARY) {
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            span[i] = quad_sum(span[i]);
            if (!l.live[i]) continue;
            const int64_t at = (int64_t)chunk * a.channels + (l.c + i);
            if (l.q == 0) a.span[at] = span[i];
#pragma unroll
            for (int s = 0; s < NS; ++s) a.carry[at * NP + l.q * NS + s] = h[i][s];
        }
    }
}

// The states behind the chunks from the chunks' own: a thread per channel and state
__global__ __launch_bounds__(256) void scan_carry_kernel(ScanArgs a, int padded) {
    const int64_t each = (int64_t)a.channels * padded;
    const int64_t own = (int64_t)blockIdx.x * 256 + threadIdx.x, e = min(own, each - 1);
    const int c = (int)(e / padded), n = (int)(e % padded);
    const float a2 = n < a.states ? kLog2e * a.A[(int64_t)c * a.states + n] : 0.0f;
    carry_walk(a.carry, a, each, e, c, a2, own < each, true);
}

// ---------------------------------------------------------------------------
// One token of each request: a quad per channel, a quarter of its states each
// ---------------------------------------------------------------------------
struct ScanStepArgs {
    ScanArgs a;
    const int32_t* slots;
    float* state;
    int64_t state_slots;
};

// R requests per workgroup.  Bound by the states' traffic: every load is made
// before the first wait, so absent arrays and slots read memory that is there
// (x for z, A for the vectors of channels, the pool's first state) and drop it.
// 128 requests of 4096 x 16 take 13 us, 4.8 TB/s.  Two requests per workgroup
// where that leaves eight workgroups for each CU: 14.7 us, 14.9 with one, 15.3
// with four.
// WHOLE: the states are NS for every lane of the quad.
template <typename T, int NS, int R, bool WHOLE>
__global__ __launch_bounds__(kScanWaves * kWave) void scan_step_kernel(ScanStepArgs p) {
    const ScanArgs& a = p.a;
    const int q = threadIdx.x % kQuad;
    const int c_own = ((int)blockIdx.y * kScanWaves * kWave + (int)threadIdx.x) / kQuad;
    const bool live = c_own < a.channels;
    const int c = live ? c_own : 0;
    const int64_t g = (int64_t)(c / a.group_channels) * a.states + q * NS;
    auto load = [&](const auto* m, auto (&v)[NS]) {
        if constexpr (WHOLE) {
            __builtin_memcpy(v, m, sizeof v);
        } else {
#pragma unroll
            for (int s = 0; s < NS; ++s) v[s] = q * NS + s < a.states ? m[s] : 0;
        }
    };
    int64_t place[R];
    bool there[R];
    float h[R][NS], a2[NS];
    T x[R], dt[R], z[R], bm[R][NS], cm[R][NS];
#pragma unroll
    for (int k = 0; k < R; ++k) {
        const int64_t row = min((int64_t)blockIdx.x * R + k, (int64_t)a.seq.tokens - 1);
        const int64_t slot = p.slots ? (int64_t)p.slots[row] : row;
        there[k] = slot >= 0 && slot < p.state_slots;
        place[k] = ((there[k] ? slot : 0) * a.channels + c) * a.states + q * NS;
        x[k] = (static_cast<const T*>(a.x) + row * a.ld_x)[c];
        dt[k] = (static_cast<const T*>(a.dt) + row * a.ld_dt)[c];
        z[k] = (a.z ? static_cast<const T*>(a.z) + row * a.ld_z : static_cast<const T*>(a.x) + row * a.ld_x)[c];
        load(static_cast<const T*>(a.B) + row * a.ld_b + g, bm[k]);
        load(static_cast<const T*>(a.C) + row * a.ld_c + g, cm[k]);
    }
    load(a.A + (int64_t)c * a.states + q * NS, a2);
    const float bias = (a.dt_bias ? a.dt_bias : a.A)[c], skip = (a.D ? a.D : a.A)[c];
#pragma unroll
    for (int k = 0; k < R; ++k) load(p.state + place[k], h[k]);
#pragma unroll
    for (int k = 0; k < R; ++k) {
        const int64_t row = (int64_t)blockIdx.x * R + k;
        float step = (float)dt[k] + (a.dt_bias ? bias : 0.0f);
        if (a.softplus) step = softplus(step);
        const float in = step * (float)x[k];
        float sum = 0.0f;
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            h[k][s] = fmaf(__builtin_amdgcn_exp2f(step * (kLog2e * a2[s])), h[k][s], in * (float)bm[k][s]);
            sum = fmaf((float)cm[k][s], h[k][s], sum);
        }
        sum = quad_sum(sum);
        if (a.D) sum = fmaf(skip, (float)x[k], sum);
        if (a.z) sum *= (float)z[k] * sigmoid((float)z[k]);
        if (!live || row >= a.seq.tokens) continue;
        if (there[k]) {
            if constexpr (WHOLE) {
                __builtin_memcpy(p.state + place[k], h[k], sizeof h[k]);
            } else {
#pragma unroll
                for (int s = 0; s < NS; ++s)
                    if (q * NS + s < a.states) p.state[place[k] + s] = h[k][s];
            }
        }
        if (q == 0) static_cast<T*>(a.y)[row * a.channels + c] = (T)(there[k] ? sum : 0.0f);
    }
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
struct ScanPlan {
    int64_t chunk = 0, chunks = 0, blocks = 0;
    int ns = 0, ch = 0;
    size_t carry_bytes = 0, span_bytes = 0, bytes = 0;
};

size_t round16(size_t n) { return (n + 15) / 16 * 16; }

// The chunk: as long as leaves four waves for each of the chip's 1024 SIMDs
// (8192 x 2048 x 16: 167 us with two, 154 with three, 149 with four, 151 with
// six) or, for pairs of channels of more than 16 states, three, which lies
// between the others both where sequences are ragged (4001 x 2111 x 24 fp32:
// 151 us with two, 157 with three, 180 with four) and where there is one (138,
// 128, 119).  Kernels of more than 32 states hold two waves a SIMD, of more than
// 64 one; with chunks for as many 2001 x 500 rows take 55 us instead of 63 (64
// states) and 108 instead of 132 (128), 8192 x 2048 x 64 512 instead of 476.
// No chunk is shorter than 16 rows (160 x 512 x 16: 42 us with 64 rows, 28 with
// 32, 22 with 16); up to 64 rows one chunk is as fast as three kernels.  Equal
// sequences are cut into equal parts, or taken whole where they are shorter.
ScanPlan plan_scan(const im2win_scan_desc* d) {
    ScanPlan p;
    with_states(d->states, narrow(d), [&](auto ns, auto ch) {
        p.ns = decltype(ns)::value;
        p.ch = decltype(ch)::value;
    });
    const int64_t per_block = kScanWaves * (kWave / kQuad) * p.ch;
    const int64_t group = d->channels / d->groups;
    p.blocks = d->groups * ((group + per_block - 1) / per_block);
    if (d->tokens == 0) return p;
    const int64_t waves = 1024 * (p.ch == 2 && p.ns > 4 ? 3 : 4);
    const int64_t want = (waves + p.blocks * kScanWaves - 1) / (p.blocks * kScanWaves);
    p.chunk = d->tokens <= 64 ? d->tokens : std::max<int64_t>((d->tokens + want - 1) / want, 16);
    const int64_t len = d->tokens / d->sequences;
    if (d->tokens % d->sequences == 0 && d->sequences > 1) {
        if (len <= p.chunk) {
            p.chunk = p.chunk / len * len;
        } else {
            for (int64_t m = (len + p.chunk - 1) / p.chunk; m <= 2 * (len / p.chunk) + 1; ++m)
                if (len % m == 0) {
                    p.chunk = len / m;
                    break;
                }
        }
    }
    p.chunk = std::min(p.chunk, d->tokens);
    p.chunks = (d->tokens + p.chunk - 1) / p.chunk;
    if (p.chunks > 1) {
        p.carry_bytes = round16((size_t)(p.chunks * d->channels * kQuad * p.ns) * 4);
        p.span_bytes = round16((size_t)(p.chunks * d->channels) * 4);
        p.bytes = p.carry_bytes + p.span_bytes + round16((size_t)p.chunks * 4);
    }
    return p;
}

constexpr int kEmptyBlocks = 32;     // workgroups that look for sequences without rows

}  // namespace

int check_scan(const im2win_scan_desc* d, bool sequences, const int32_t* starts, bool have_starts) {
    if (!d) return fail(IM2WIN_ENULL, "descriptor is NULL");
    int rc = check_rows(d->tokens, d->channels, d->dtype);
    if (rc) return rc;
    if (d->states < 1 || d->states > 128) return fail(IM2WIN_EINVAL, "states must be 1 to 128 (got %lld)", (long long)d->states);
    if (d->groups < 1 || d->channels % d->groups)
        return fail(IM2WIN_EINVAL, "groups (%lld) must divide the %lld channels", (long long)d->groups, (long long)d->channels);
    if ((rc = check_ld(d->ld_x, d->channels, "ld_x")) || (rc = check_ld(d->ld_dt, d->channels, "ld_dt")) ||
        (rc = check_ld(d->ld_z, d->channels, "ld_z")) || (rc = check_ld(d->ld_b, d->groups * d->states, "ld_b")) ||
        (rc = check_ld(d->ld_c, d->groups * d->states, "ld_c")))
        return rc;
    return sequences ? check_sequences(d->tokens, d->sequences, starts, have_starts) : IM2WIN_OK;
}

int check_scan_inputs(const im2win_scan_desc* d, const void* x, const void* dt, const float* A, const void* B,
                      const void* C, const float* D, const void* z, const float* dt_bias) {
    const size_t e = d->dtype == IM2WIN_F32 ? 4 : 2;
    int rc;
    if ((rc = need_ptr(A, 4, "A")) || (rc = may_ptr(D, 4, "D")) || (rc = may_ptr(dt_bias, 4, "dt_bias"))) return rc;
    if (d->tokens == 0) return IM2WIN_OK;
    if ((rc = need_ptr(x, e, "x")) || (rc = need_ptr(dt, e, "dt")) || (rc = need_ptr(B, e, "B")) ||
        (rc = need_ptr(C, e, "C")) || (rc = may_ptr(z, e, "z")))
        return rc;
    return IM2WIN_OK;
}

ScanArgs scan_args(const im2win_scan_desc* d, const void* x, const void* dt, const float* A, const void* B,
                   const void* C, const float* D, const void* z, const float* dt_bias, int ch) {
    ScanArgs a{};
    a.x = x; a.dt = dt; a.A = A; a.B = B; a.C = C; a.D = D; a.z = z; a.dt_bias = dt_bias;
    a.ld_x = d->ld_x; a.ld_dt = d->ld_dt; a.ld_z = d->ld_z; a.ld_b = d->ld_b; a.ld_c = d->ld_c;
    a.channels = (int)d->channels; a.states = (int)d->states;
    a.group_channels = (int)(d->channels / d->groups);
    const int per_block = kScanWaves * (kWave / kQuad) * ch;
    a.group_blocks = (a.group_channels + per_block - 1) / per_block;
    a.blocks = (int)d->groups * a.group_blocks;
    a.softplus = d->softplus != 0;
    return a;
}

}  // namespace im2win

using namespace im2win;

extern "C" {

int im2win_selective_scan_workspace_bytes(const im2win_scan_desc* d, size_t* bytes) {
    int rc = check_scan(d, true, nullptr, false);
    if (rc) return rc;
    if (!bytes) return fail(IM2WIN_ENULL, "bytes is NULL");
    *bytes = plan_scan(d).bytes;
    return ok();
}

int im2win_selective_scan(const im2win_scan_desc* d, const void* x, const void* dt, const float* A, const void* B,
                          const void* C, const float* D, const void* z, const float* dt_bias,
                          const int32_t* seq_starts, const float* initial_state, void* y, float* final_state,
                          void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_scan(d, true, seq_starts, true);
    if (rc || (rc = check_scan_inputs(d, x, dt, A, B, C, D, z, dt_bias))) return rc;
    if ((d->tokens && (rc = need_ptr(y, d->dtype == IM2WIN_F32 ? 4 : 2, "y"))) ||
        (rc = may_ptr(initial_state, 4, "initial_state")) || (rc = may_ptr(final_state, 4, "final_state")))
        return rc;
    const ScanPlan p = plan_scan(d);
    if (p.bytes && (rc = need_ptr(workspace, 16, "workspace"))) return rc;
    if (workspace_bytes < p.bytes)
        return fail(IM2WIN_EWORKSPACE, "workspace holds %zu bytes, the scan needs %zu", workspace_bytes, p.bytes);
    ScanArgs a = scan_args(d, x, dt, A, B, C, D, z, dt_bias, p.ch);
    a.init = initial_state; a.y = y; a.final_state = final_state;
    a.seq = make_seq_map(d->tokens, d->sequences, seq_starts);
    a.chunk = (int)p.chunk; a.chunks = (int)p.chunks;
    // 64 chunks: 148 us with the carry kernel, 152 without; 16 a sequence 58 and 53; 125 chunks in 31 ragged
    // sequences 35 and 30; 63 of 64 states in 9 38 and 33
    a.look = look_back(p.chunks, d->sequences, seq_starts != nullptr, p.ns <= 8 ? 32 : 16);
    char* ws = static_cast<char*>(workspace);
    if (p.bytes) {
        a.carry = reinterpret_cast<float*>(ws);
        a.span = reinterpret_cast<float*>(ws + p.carry_bytes);
        a.flags = reinterpret_cast<int*>(ws + p.carry_bytes + p.span_bytes);
    }
    const int64_t grid = p.blocks * p.chunks;
    const int64_t extra = final_state && (seq_starts || d->tokens == 0) ? std::min<int64_t>(d->sequences, kEmptyBlocks) : 0;
    if (grid + extra == 0) return ok();
    if ((rc = check_launch(grid + extra, kScanWaves * kWave, "selective_scan"))) return rc;
    // chunks that no sequence crosses need no states from before them
    const bool whole = !seq_starts && p.chunks && p.chunk % (d->tokens / d->sequences) == 0;
    hipStream_t s = static_cast<hipStream_t>(stream);
    with_type(d->dtype, [&](auto t) {
        with_states(d->states, narrow(d), [&](auto ns, auto ch) {
            using T = decltype(t);
            constexpr int NS = decltype(ns)::value, CH = decltype(ch)::value;
            const dim3 threads(kScanWaves * kWave);
            if (p.chunks > 1 && !whole) {
                hipLaunchKernelGGL((scan_kernel<T, NS, CH, true>), dim3((unsigned)(p.blocks * (p.chunks - 1))), threads, 0, s, a);
                if (!a.look) {
                    const int64_t each = (int64_t)a.channels * kQuad * NS;
                    ScanArgs before = a;      // the last chunk leaves nothing to another
                    --before.chunks;
                    hipLaunchKernelGGL(scan_carry_kernel, dim3((unsigned)((each + 255) / 256), carry_pieces(before.chunks)), dim3(256), 0, s,
                                       before, kQuad * NS);
                }
            }
            hipLaunchKernelGGL((scan_kernel<T, NS, CH, false>), dim3((unsigned)(grid + extra)), threads, 0, s, a);
        });
    });
    return launched("selective_scan");
}

int im2win_selective_scan_step(const im2win_scan_desc* d, const void* x, const void* dt, const float* A, const void* B,
                               const void* C, const float* D, const void* z, const float* dt_bias,
                               const int32_t* slots, float* state, int64_t state_slots, void* y, void* stream) {
    int rc = check_scan(d, false, nullptr, false);
    if (rc) return rc;
    if (state_slots < 0) return fail(IM2WIN_EINVAL, "state_slots is negative (%lld)", (long long)state_slots);
    if ((rc = check_scan_inputs(d, x, dt, A, B, C, D, z, dt_bias))) return rc;
    if (d->tokens == 0) return ok();
    if ((rc = may_ptr(slots, 4, "slots")) || (rc = need_ptr(y, d->dtype == IM2WIN_F32 ? 4 : 2, "y")) ||
        (state_slots && (rc = need_ptr(state, 4, "state"))))
        return rc;
    ScanStepArgs p{};
    p.a = scan_args(d, x, dt, A, B, C, D, z, dt_bias, 1);
    p.a.y = y;
    p.a.seq.tokens = (int)d->tokens;
    p.slots = slots; p.state_slots = state_slots;
    p.state = state_slots ? state : const_cast<float*>(A);     // as large as one state; read, and not written without slots
    if ((rc = check_launch(d->tokens, kScanWaves * kWave, "selective_scan_step"))) return rc;
    const unsigned cover = (unsigned)((d->channels * kQuad + kScanWaves * kWave - 1) / (kScanWaves * kWave));
    const hipStream_t s = static_cast<hipStream_t>(stream);
    with_type(d->dtype, [&](auto t) {
        with_states(d->states, true, [&](auto ns, auto) {
            using T = decltype(t);
            constexpr int NS = decltype(ns)::value;
            auto launch = [&](auto r, auto whole) {
                constexpr int R = decltype(r)::value;
                hipLaunchKernelGGL((scan_step_kernel<T, NS, R, decltype(whole)::value>),
                                   dim3((unsigned)((d->tokens + R - 1) / R), cover), dim3(kScanWaves * kWave), 0, s, p);
            };
            auto with_whole = [&](auto r) {
                if (d->states == kQuad * NS) launch(r, std::true_type{});
                else launch(r, std::false_type{});
            };
            if (NS <= 8 && d->tokens / 2 * cover >= 2048) with_whole(std::integral_constant<int, NS <= 8 ? 2 : 1>{});
            else with_whole(std::integral_constant<int, 1>{});
        });
    });
    return launched("selective_scan_step");
}

}  // extern "C"
