// Short causal convolution (im2win_causal_conv1d*, include/im2win_seq.h): a
// depthwise convolution along time over packed sequences of token rows.
#include <algorithm>

#include "seq_common.h"

namespace im2win {
namespace {

struct Conv1dArgs {
    const void* x;
    const void* w;
    const void* bias;
    const void* init;
    void* y;
    void* final_state;
    SeqMap seq;
    int64_t ld_x;
    int channels;
    int tiles;          // token tiles; tiles behind them write final states
    int groups;         // workgroups beside one another that cover a row
    int silu;
};

// Tokens per wave.  Short tiles read their W-1 rows of overlap from L2 again
// but fill the chip: 16384 x 4096 bf16 (4 taps) takes 62 us with 16 rows, 50
// with 8, 51 with 4, and 512 x 512 takes 14.7, 8.5 and 8.4.
constexpr int kConvTile = 4;
constexpr int kConvWaves = 4;    // waves per workgroup, each with its own tile

template <typename T, int V, int W>
struct Taps {
    float w[W][V];
    float bias[V];

    __device__ void load(const T* wp, const T* bp, int c) {
        float flat[W][V];
#pragma unroll
        for (int i = 0; i < W; ++i) load_vec<V>(wp + (int64_t)c * W + i * V, flat[i]);
#pragma unroll
        for (int k = 0; k < W; ++k)
#pragma unroll
            for (int v = 0; v < V; ++v) w[k][v] = flat[(v * W + k) / V][(v * W + k) % V];
        if (bp) load_vec<V>(bp + c, bias);
        else
#pragma unroll
            for (int v = 0; v < V; ++v) bias[v] = 0.0f;
    }
};

// The input `back` rows before row t of a sequence whose first row is
// `first`: a row of x, a row of the sequence's initial state, or zero.
template <typename T, int V, int W>
__device__ __forceinline__ void load_input(const T* x, const T* init, int64_t ld, int channels, int b, int first,
                                           int t, int back, int c, float (&v)[V]) {
    const int p = t - back - first;
    if (p >= 0) {
        load_vec<V>(x + (int64_t)(t - back) * ld + c, v);
    } else if (init) {
        load_vec<V>(init + ((int64_t)b * (W - 1) + (W - 1 + p)) * channels + c, v);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = 0.0f;
    }
}

// The first of a lane's V channels, and whether the lane stores anything.  A
// last lane with fewer than V channels of its own takes the row's last V (two
// lanes then compute and store the same values); lanes past it read them only.
template <int V>
__device__ __forceinline__ bool lane_channels(int group, int lane, int channels, int* c) {
    const int own = (group * kWave + lane) * V;
    *c = min(own, channels - V);
    return own < channels;
}

// One wave: kConvTile rows of 64*V channels.  Bound by memory: each wave has
// all its rows' loads in flight before it uses the first.  16384 x 4096 bf16
// of four taps: 52 us, 5.2 TB/s for x read and y written once.
template <typename T, int V, int W>
__global__ __launch_bounds__(kConvWaves * kWave) void conv1d_kernel(Conv1dArgs a) {
    const T* x = static_cast<const T*>(a.x);
    const T* init = static_cast<const T*>(a.init);
    T* y = static_cast<T*>(a.y);
    const int64_t tile = (int64_t)(blockIdx.x / a.groups) * kConvWaves + uniform(threadIdx.x / kWave);
    int c;
    const bool live = lane_channels<V>(blockIdx.x % a.groups, threadIdx.x % kWave, a.channels, &c);

    if (tile >= a.tiles) {
        // one row of a final state: input e of the sequence with its W-1 earlier ones in front
        if constexpr (W > 1) {
            const int64_t row = tile - a.tiles;
            if (!a.final_state || row >= (int64_t)a.seq.count * (W - 1)) return;
            const int b = (int)(row / (W - 1)), j = (int)(row % (W - 1));
            const int first = a.seq.first(b), end = max(a.seq.first(b + 1), first);
            float v[V];
            load_input<T, V, W>(x, init, a.ld_x, a.channels, b, first, end, W - 1 - j, c, v);
            if (live) store_vec<V>(static_cast<T*>(a.final_state) + row * a.channels + c, v);
        }
        return;
    }

    const int t0 = (int)tile * kConvTile;
    const int lo = max(a.seq.first(0), t0), hi = min(a.seq.first(a.seq.count), t0 + kConvTile);
    if (lo >= hi) return;
    Taps<T, V, W> taps;
    taps.load(static_cast<const T*>(a.w), static_cast<const T*>(a.bias), c);
    SeqMap::Found in_seq = a.seq.at(lo);

    auto finish = [&](int t, float (&acc)[V]) {
        if (a.silu)
#pragma unroll
            for (int v = 0; v < V; ++v) acc[v] *= sigmoid(acc[v]);
        if (live) store_vec<V>(y + (int64_t)t * a.channels + c, acc);
    };

    if (lo == t0 && hi == t0 + kConvTile && in_seq.end >= hi && lo - in_seq.first >= W - 1) {
        // the tile and the rows before it lie in one sequence
        Bits<T, V> in[kConvTile + W - 1];
        const T* p = x + (int64_t)(t0 - (W - 1)) * a.ld_x + c;
#pragma unroll
        for (int i = 0; i < kConvTile + W - 1; ++i, p += a.ld_x) in[i].load(p);
#pragma unroll
        for (int i = 0; i < kConvTile; ++i) {
            float acc[V];
#pragma unroll
            for (int v = 0; v < V; ++v) {
                acc[v] = taps.bias[v];
#pragma unroll
                for (int k = 0; k < W; ++k) acc[v] = fmaf(taps.w[k][v], in[i + k].get(v), acc[v]);
            }
            finish(t0 + i, acc);
        }
        return;
    }
    for (int t = lo; t < hi; ++t) {
        if (t >= in_seq.end) in_seq = a.seq.at(t);
        float acc[V];
#pragma unroll
        for (int v = 0; v < V; ++v) acc[v] = taps.bias[v];
#pragma unroll
        for (int k = 0; k < W; ++k) {
            float in[V];
            load_input<T, V, W>(x, init, a.ld_x, a.channels, in_seq.b, in_seq.first, t, W - 1 - k, c, in);
#pragma unroll
            for (int v = 0; v < V; ++v) acc[v] = fmaf(taps.w[k][v], in[v], acc[v]);
        }
        finish(t, acc);
    }
}

// ---------------------------------------------------------------------------
// Gradients.  With s the sum in front of the activation and g = dy act'(s),
//   dx[t] = sum_k w[k] g[t + W-1 - k]  (rows of the same sequence)
//   dw[k] = sum_t g[t] x[t - (W-1) + k],  dbias = sum_t g[t].
// One wave walks a stripe of rows and the W-1 rows behind it, with the last W
// inputs and gradients in registers; the stripes' sums of dw and dbias go to
// the workspace, one row of (W+1) x D for each workgroup, and a second kernel
// adds them in order.  16384 x 4096 bf16 of four taps: 91 us, 4.4 TB/s for x,
// dy and dx; 80% of the issue slots are taken (s again, its sigmoid, and three
// sums of W products an element).
// ---------------------------------------------------------------------------
struct Conv1dBwdArgs {
    const void* dy;
    const void* x;
    const void* w;
    const void* bias;
    const void* init;
    const void* d_final;
    void* dx;
    void* d_init;
    float* part;        // [parts][W + 1][channels]
    float* dw;
    float* dbias;
    SeqMap seq;
    int64_t ld_x;
    int channels;
    int groups;
    int silu;
    int stripe;         // rows per wave
    int parts;
};

constexpr int kConvBatch = 4;     // rows in flight

// Rows per wave: a walk of a stripe is serial, so a short problem takes short
// stripes, and a large one long ones, whose sums are fewer: the longest that
// leaves a wave for each of the chip's 1024 SIMDs.  16384 x 4096 bf16 takes 91
// us with 64 rows, 98 with 32 and 110 with 16; 512 x 512 takes 44, 26 and 17.5
// with 64, 32 and 8; 8000 x 2001 fp32 takes 63, 56 and 62 with 64, 32 and 16.
int64_t stripe_of(int64_t tokens, int64_t groups) {
    int64_t stripe = 64;
    while (stripe > 8 && groups * ((tokens + stripe - 1) / stripe) < 1024) stripe /= 2;
    return stripe;
}

template <int V>
__device__ __forceinline__ void times_slope(float (&g)[V], const float (&s)[V], int silu) {
    if (silu)
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const float sig = sigmoid(s[v]);
            g[v] *= sig * fmaf(s[v], 1.0f - sig, 1.0f);
        }
}

template <typename T, int V, int W>
__global__ __launch_bounds__(kConvWaves * kWave) void conv1d_bwd_kernel(Conv1dBwdArgs a) {
    __shared__ float sum[kConvWaves][kWave][V + 1];
    const T* x = static_cast<const T*>(a.x);
    const T* dy = static_cast<const T*>(a.dy);
    const T* init = static_cast<const T*>(a.init);
    const T* d_final = static_cast<const T*>(a.d_final);
    T* dx = static_cast<T*>(a.dx);
    const int wave = uniform(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    int c;
    const bool live = lane_channels<V>(blockIdx.x % a.groups, lane, a.channels, &c);
    const int part = blockIdx.x / a.groups;

    Taps<T, V, W> taps;
    taps.load(static_cast<const T*>(a.w), static_cast<const T*>(a.bias), c);
    float dw[W + 1][V] = {};                 // the last row is dbias

    const int64_t s0 = ((int64_t)part * kConvWaves + wave) * a.stripe;
    const int lo = (int)max<int64_t>(a.seq.first(0), s0);
    const int hi = (int)min<int64_t>(a.seq.first(a.seq.count), s0 + a.stripe);
    for (int t = lo; t < hi;) {
        const SeqMap::Found in_seq = a.seq.at(t);
        const int b = in_seq.b, first = in_seq.first, end = max(in_seq.end, t + 1);
        const int own = min(end, hi);        // rows [t, own) of this sequence are the stripe's
        float win[W][V], g[W][V] = {};
#pragma unroll
        for (int j = 0; j < W - 1; ++j)
            load_input<T, V, W>(x, init, a.ld_x, a.channels, b, first, t, W - 1 - j, c, win[j]);

        // g of row r, with its window; r's own sums where `mine`
        auto row = [&](const Bits<T, V>& xr, const Bits<T, V>& dyr, bool mine) {
            float s[V];
#pragma unroll
            for (int v = 0; v < V; ++v) {
                win[W - 1][v] = xr.get(v);
                g[W - 1][v] = dyr.get(v);
                s[v] = taps.bias[v];
#pragma unroll
                for (int k = 0; k < W; ++k) s[v] = fmaf(taps.w[k][v], win[k][v], s[v]);
            }
            times_slope<V>(g[W - 1], s, a.silu);
            if (mine) {
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    dw[W][v] += g[W - 1][v];
#pragma unroll
                    for (int k = 0; k < W; ++k) dw[k][v] = fmaf(g[W - 1][v], win[k][v], dw[k][v]);
                }
            }
#pragma unroll
            for (int k = 0; k + 1 < W; ++k)
#pragma unroll
                for (int v = 0; v < V; ++v) win[k][v] = win[k + 1][v];
        };
        auto shift = [&]() {
#pragma unroll
            for (int k = 0; k + 1 < W; ++k)
#pragma unroll
                for (int v = 0; v < V; ++v) g[k][v] = g[k + 1][v];
        };
        // dx of row u, whose gradient and the W-1 behind it are in g
        auto input_grad = [&](int u, float (&d)[V]) {
#pragma unroll
            for (int v = 0; v < V; ++v) d[v] = 0.0f;
            if (d_final && u >= t && u >= end - (W - 1))
                load_vec<V>(d_final + ((int64_t)b * (W - 1) + (u - (end - (W - 1)))) * a.channels + c, d);
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int k = 0; k < W; ++k) d[v] = fmaf(taps.w[k][v], g[W - 1 - k][v], d[v]);
        };
        auto put = [&](int u, const float (&d)[V]) {
            if (u >= t && live) store_vec<V>(dx + (int64_t)u * a.channels + c, d);
        };

        // the stripe's rows and the W-1 behind, which its last ones reach: kConvBatch rows are loaded
        // while the ones before them are worked on
        const int reach = min(own + W - 1, end);
        Bits<T, V> nx[kConvBatch], ng[kConvBatch];
        auto fetch = [&](int r) {
#pragma unroll
            for (int i = 0; i < kConvBatch; ++i) {
                const int64_t at = min(r + i, reach - 1);
                nx[i].load(x + at * a.ld_x + c);
                ng[i].load(dy + at * a.channels + c);
            }
        };
        fetch(t);
        for (int r = t; r < reach; r += kConvBatch) {
            Bits<T, V> cx[kConvBatch], cg[kConvBatch];
#pragma unroll
            for (int i = 0; i < kConvBatch; ++i) {
                cx[i] = nx[i];
                cg[i] = ng[i];
            }
            if (r + kConvBatch < reach) fetch(r + kConvBatch);
            float d[kConvBatch][V];
#pragma unroll
            for (int i = 0; i < kConvBatch; ++i) {
                if (r + i >= reach) break;
                shift();
                row(cx[i], cg[i], r + i < own);
                input_grad(r + i - (W - 1), d[i]);
            }
#pragma unroll
            for (int i = 0; i < kConvBatch; ++i) {
                nx[i].wait();
                ng[i].wait();
            }
#pragma unroll
            for (int i = 0; i < kConvBatch; ++i)
                if (r + i < reach) put(r + i - (W - 1), d[i]);
        }
        // behind the sequence's end there is no gradient
        for (int r = reach; r < own + W - 1; ++r) {
            shift();
#pragma unroll
            for (int v = 0; v < V; ++v) g[W - 1][v] = 0.0f;
            float d[V];
            input_grad(r - (W - 1), d);
            put(r - (W - 1), d);
        }
        t = own;
    }

    // the workgroup's sums, wave after wave
#pragma unroll
    for (int k = 0; k <= W; ++k) {
        __syncthreads();
#pragma unroll
        for (int v = 0; v < V; ++v) sum[wave][lane][v] = dw[k][v];
        __syncthreads();
        if (wave == 0 && live) {
            float s[V];
#pragma unroll
            for (int v = 0; v < V; ++v) {
                s[v] = sum[0][lane][v];
#pragma unroll
                for (int i = 1; i < kConvWaves; ++i) s[v] += sum[i][lane][v];
            }
            store_vec<V>(a.part + ((int64_t)part * (W + 1) + k) * a.channels + c, s);
        }
    }
}

constexpr int kSumWaves = 8;

// What is left after the walks, one workgroup for each row of 512 channels
// that a state's gradient has, and before them one for each 64 channels of a
// tap (or of the bias): its workgroups' sums, every eighth per wave, eight
// loads in flight.
template <typename T, int W>
__global__ __launch_bounds__(kSumWaves * kWave) void conv1d_bwd_finish_kernel(Conv1dBwdArgs a) {
    __shared__ float sum[kSumWaves][kWave];
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    const int across = (a.channels + kWave - 1) / kWave;
    if ((int64_t)blockIdx.x < (int64_t)across * (W + 1)) {
        const int c = (int)(blockIdx.x % across) * kWave + lane, k = blockIdx.x / across;
        float s = 0.0f;
        if (c < a.channels) {
#pragma unroll 8
            for (int i = wave; i < a.parts; i += kSumWaves)
                s += a.part[((int64_t)i * (W + 1) + k) * a.channels + c];
        }
        sum[wave][lane] = s;
        __syncthreads();
        if (wave == 0 && c < a.channels) {
#pragma unroll
            for (int i = 1; i < kSumWaves; ++i) s += sum[i][lane];
            if (k < W) a.dw[(int64_t)c * W + k] = s;
            else if (a.dbias) a.dbias[c] = s;
        }
        return;
    }
    if constexpr (W > 1) {
        // row e of a sequence's W-1 earlier inputs
        const T* x = static_cast<const T*>(a.x);
        const T* init = static_cast<const T*>(a.init);
        const T* d_final = static_cast<const T*>(a.d_final);
        const int wide = (a.channels + kSumWaves * kWave - 1) / (kSumWaves * kWave);
        const int64_t block = (int64_t)blockIdx.x - (int64_t)across * (W + 1), row = block / wide;
        const int b = (int)(row / (W - 1)), e = (int)(row % (W - 1));
        const int first = a.seq.first(b), end = max(a.seq.first(b + 1), first), len = end - first;
        const int c = (int)(block % wide) * kSumWaves * kWave + threadIdx.x;
        if (c >= a.channels) return;
        Taps<T, 1, W> taps;
        taps.load(static_cast<const T*>(a.w), static_cast<const T*>(a.bias), c);
        float d = 0.0f;
        if (d_final && e >= len) d = (float)d_final[((int64_t)b * (W - 1) + (e - len)) * a.channels + c];
#pragma unroll
        for (int k = 0; k < W; ++k) {
            const int p = e - k;             // the row of the sequence that reads input e with tap k
            if (p < 0 || p >= len) continue;
            float s[1] = {taps.bias[0]}, g[1] = {(float)static_cast<const T*>(a.dy)[(int64_t)(first + p) * a.channels + c]};
#pragma unroll
            for (int j = 0; j < W; ++j) {
                float in[1];
                load_input<T, 1, W>(x, init, a.ld_x, a.channels, b, first, first + p, W - 1 - j, c, in);
                s[0] = fmaf(taps.w[j][0], in[0], s[0]);
            }
            times_slope<1>(g, s, a.silu);
            d = fmaf(taps.w[k][0], g[0], d);
        }
        static_cast<T*>(a.d_init)[row * a.channels + c] = (T)d;
    }
}

// ---------------------------------------------------------------------------
// One token of each request: the W-1 kept inputs move up by one.  16 requests
// of 2048 channels take 3.3 us, a launch and two dependent loads.
// ---------------------------------------------------------------------------
struct Conv1dStepArgs {
    const void* x;
    const void* w;
    const void* bias;
    const int32_t* slots;
    void* state;
    void* y;
    int64_t state_slots;
    int64_t ld_x;
    int channels;
    int silu;
};

template <typename T, int V, int W>
__global__ __launch_bounds__(kWave) void conv1d_step_kernel(Conv1dStepArgs a) {
    const int64_t row = blockIdx.x;
    const int c = ((int)blockIdx.y * kWave + (int)threadIdx.x) * V;
    if (c >= a.channels) return;
    T* y = static_cast<T*>(a.y) + row * a.channels + c;
    const int64_t slot = a.slots ? (int64_t)a.slots[row] : row;
    float acc[V] = {};
    if (slot < 0 || slot >= a.state_slots) {
        store_vec<V>(y, acc);
        return;
    }
    Taps<T, V, W> taps;
    taps.load(static_cast<const T*>(a.w), static_cast<const T*>(a.bias), c);
    T* state = static_cast<T*>(a.state) + slot * (W - 1) * a.channels + c;
    float win[W][V];
#pragma unroll
    for (int j = 0; j < W - 1; ++j) load_vec<V>(state + (int64_t)j * a.channels, win[j]);
    load_vec<V>(static_cast<const T*>(a.x) + row * a.ld_x + c, win[W - 1]);
#pragma unroll
    for (int v = 0; v < V; ++v) {
        acc[v] = taps.bias[v];
#pragma unroll
        for (int k = 0; k < W; ++k) acc[v] = fmaf(taps.w[k][v], win[k][v], acc[v]);
        if (a.silu) acc[v] *= sigmoid(acc[v]);
    }
#pragma unroll
    for (int j = 0; j < W - 1; ++j) store_vec<V>(state + (int64_t)j * a.channels, win[j + 1]);
    store_vec<V>(y, acc);
}

// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
int check_desc(const im2win_conv1d_desc* d) {
    if (!d) return fail(IM2WIN_ENULL, "descriptor is NULL");
    int rc = check_rows(d->tokens, d->channels, d->dtype);
    if (rc) return rc;
    if (d->width < 1 || d->width > 8) return fail(IM2WIN_EINVAL, "width must be 1 to 8 (got %lld)", (long long)d->width);
    return check_ld(d->ld_x, d->channels, "ld_x");
}

size_t elem_of(const im2win_conv1d_desc* d) { return d->dtype == IM2WIN_F32 ? 4 : 2; }

// Lanes of 16 bytes each need as many channels; the step, which reads and
// writes its state in place, also that no two lanes share a channel.
bool vectors(const im2win_conv1d_desc* d) { return d->channels * elem_of(d) >= 16; }
bool whole_vectors(const im2win_conv1d_desc* d) { return d->channels * elem_of(d) % 16 == 0; }

int64_t channel_groups(int64_t channels, int v) { return (channels + kWave * v - 1) / (kWave * v); }

struct BwdPlan {
    int64_t groups, stripe, parts;
    size_t bytes;
};

BwdPlan plan_bwd(const im2win_conv1d_desc* d) {
    BwdPlan p;
    p.groups = channel_groups(d->channels, vectors(d) ? (int)(16 / elem_of(d)) : 1);
    p.stripe = stripe_of(d->tokens, p.groups);
    p.parts = (d->tokens + p.stripe * kConvWaves - 1) / (p.stripe * kConvWaves);
    p.bytes = (size_t)(p.parts * (d->width + 1) * d->channels * 4);
    return p;
}

template <typename F>
void with_width(int64_t w, F f) {
    switch (w) {
        case 1: f(std::integral_constant<int, 1>{}); break;
        case 2: f(std::integral_constant<int, 2>{}); break;
        case 3: f(std::integral_constant<int, 3>{}); break;
        case 4: f(std::integral_constant<int, 4>{}); break;
        case 5: f(std::integral_constant<int, 5>{}); break;
        case 6: f(std::integral_constant<int, 6>{}); break;
        case 7: f(std::integral_constant<int, 7>{}); break;
        default: f(std::integral_constant<int, 8>{}); break;
    }
}

// f(type, vector width, taps) for the call's element type, channels and width
template <typename F>
void with_kernel(const im2win_conv1d_desc* d, bool vec, F f) {
    with_width(d->width, [&](auto w) {
        if (d->dtype == IM2WIN_F32) {
            if (vec) f(float{}, std::integral_constant<int, kVec<float>>{}, w);
            else f(float{}, std::integral_constant<int, 1>{}, w);
        } else {
            if (vec) f(bf16{}, std::integral_constant<int, kVec<bf16>>{}, w);
            else f(bf16{}, std::integral_constant<int, 1>{}, w);
        }
    });
}

}  // namespace
}  // namespace im2win

using namespace im2win;

extern "C" {

int im2win_causal_conv1d(const im2win_conv1d_desc* d, const void* x, const void* w, const void* bias,
                         const int32_t* seq_starts, const void* initial_state, void* y, void* final_state,
                         void* stream) {
    int rc = check_desc(d);
    if (rc || (rc = check_sequences(d->tokens, d->sequences, seq_starts, true))) return rc;
    const size_t e = elem_of(d);
    if (d->tokens && ((rc = need_ptr(x, e, "x")) || (rc = need_ptr(y, e, "y")))) return rc;
    if ((rc = need_ptr(w, e, "w")) || (rc = may_ptr(bias, e, "bias")) ||
        (rc = may_ptr(initial_state, e, "initial_state")) || (rc = may_ptr(final_state, e, "final_state")))
        return rc;
    Conv1dArgs a{};
    a.x = x; a.w = w; a.bias = bias; a.init = initial_state; a.y = y; a.final_state = final_state;
    a.seq = make_seq_map(d->tokens, d->sequences, seq_starts);
    a.ld_x = d->ld_x; a.channels = (int)d->channels; a.silu = d->silu != 0;
    a.tiles = (int)((d->tokens + kConvTile - 1) / kConvTile);
    const int64_t rows = a.tiles + (final_state ? d->sequences * (d->width - 1) : 0);
    if (rows == 0) return ok();
    const int64_t blocks = (rows + kConvWaves - 1) / kConvWaves;
    const bool vec = vectors(d);
    a.groups = (int)channel_groups(d->channels, vec ? (int)(16 / e) : 1);
    if ((rc = check_launch(blocks * a.groups, kConvWaves * kWave, "causal_conv1d"))) return rc;
    with_kernel(d, vec, [&](auto t, auto v, auto taps) {
        using T = decltype(t);
        constexpr int V = decltype(v)::value, W = decltype(taps)::value;
        hipLaunchKernelGGL((conv1d_kernel<T, V, W>), dim3((unsigned)(blocks * a.groups)), dim3(kConvWaves * kWave), 0,
                           static_cast<hipStream_t>(stream), a);
    });
    return launched("causal_conv1d");
}

int im2win_causal_conv1d_backward_workspace_bytes(const im2win_conv1d_desc* d, size_t* bytes) {
    int rc = check_desc(d);
    if (rc || (rc = check_sequences(d->tokens, d->sequences, nullptr, false))) return rc;
    if (!bytes) return fail(IM2WIN_ENULL, "bytes is NULL");
    *bytes = plan_bwd(d).bytes;
    return ok();
}

int im2win_causal_conv1d_backward(const im2win_conv1d_desc* d, const void* dy, const void* x, const void* w,
                                  const void* bias, const int32_t* seq_starts, const void* initial_state,
                                  const void* d_final_state, void* dx, float* dw, float* dbias,
                                  void* d_initial_state, void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_desc(d);
    if (rc || (rc = check_sequences(d->tokens, d->sequences, seq_starts, true))) return rc;
    const size_t e = elem_of(d);
    if (d->tokens && ((rc = need_ptr(dy, e, "dy")) || (rc = need_ptr(x, e, "x")) || (rc = need_ptr(dx, e, "dx")) ||
                      (rc = need_ptr(workspace, 16, "workspace"))))
        return rc;
    if ((rc = need_ptr(w, e, "w")) || (rc = need_ptr(dw, 4, "dw")) || (rc = may_ptr(bias, e, "bias")) ||
        (rc = may_ptr(dbias, 4, "dbias")) || (rc = may_ptr(initial_state, e, "initial_state")) ||
        (rc = may_ptr(d_final_state, e, "d_final_state")) || (rc = may_ptr(d_initial_state, e, "d_initial_state")))
        return rc;
    const BwdPlan p = plan_bwd(d);
    if (workspace_bytes < p.bytes)
        return fail(IM2WIN_EWORKSPACE, "workspace holds %zu bytes, the gradients need %zu", workspace_bytes, p.bytes);
    const int64_t sums = (d->channels + kWave - 1) / kWave * (d->width + 1);
    const int64_t states = d_initial_state ? d->sequences * (d->width - 1) * ((d->channels + kSumWaves * kWave - 1) / (kSumWaves * kWave)) : 0;
    if ((rc = check_launch(p.parts * p.groups, kConvWaves * kWave, "causal_conv1d_backward")) ||
        (rc = check_launch(sums + states, kSumWaves * kWave, "causal_conv1d_backward")))
        return rc;
    Conv1dBwdArgs a{};
    a.dy = dy; a.x = x; a.w = w; a.bias = bias; a.init = initial_state; a.d_final = d_final_state;
    a.dx = dx; a.d_init = d_initial_state; a.part = static_cast<float*>(workspace); a.dw = dw; a.dbias = dbias;
    a.seq = make_seq_map(d->tokens, d->sequences, seq_starts);
    a.ld_x = d->ld_x; a.channels = (int)d->channels; a.silu = d->silu != 0; a.parts = (int)p.parts;
    a.groups = (int)p.groups; a.stripe = (int)p.stripe;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const bool vec = vectors(d);
    with_kernel(d, vec, [&](auto t, auto v, auto taps) {
        using T = decltype(t);
        constexpr int V = decltype(v)::value, W = decltype(taps)::value;
        if (p.parts)
            hipLaunchKernelGGL((conv1d_bwd_kernel<T, V, W>), dim3((unsigned)(p.parts * p.groups)),
                               dim3(kConvWaves * kWave), 0, s, a);
    });
    with_kernel(d, false, [&](auto t, auto, auto taps) {
        hipLaunchKernelGGL((conv1d_bwd_finish_kernel<decltype(t), decltype(taps)::value>), dim3((unsigned)(sums + states)),
                           dim3(kSumWaves * kWave), 0, s, a);
    });
    return launched("causal_conv1d_backward");
}

int im2win_causal_conv1d_step(const im2win_conv1d_desc* d, const void* x, const void* w, const void* bias,
                              const int32_t* slots, void* state, int64_t state_slots, void* y, void* stream) {
    int rc = check_desc(d);
    if (rc) return rc;
    if (state_slots < 0) return fail(IM2WIN_EINVAL, "state_slots is negative (%lld)", (long long)state_slots);
    if (d->tokens == 0) return ok();
    const size_t e = elem_of(d);
    if ((rc = need_ptr(x, e, "x")) || (rc = need_ptr(w, e, "w")) || (rc = may_ptr(bias, e, "bias")) ||
        (rc = may_ptr(slots, 4, "slots")) || (rc = need_ptr(y, e, "y")))
        return rc;
    if (d->width > 1 && state_slots && (rc = need_ptr(state, e, "state"))) return rc;
    if ((rc = check_launch(d->tokens, kWave, "causal_conv1d_step"))) return rc;
    Conv1dStepArgs a{};
    a.x = x; a.w = w; a.bias = bias; a.slots = slots; a.state = state; a.y = y; a.state_slots = state_slots;
    a.ld_x = d->ld_x; a.channels = (int)d->channels; a.silu = d->silu != 0;
    const bool vec = whole_vectors(d);
    with_kernel(d, vec, [&](auto t, auto v, auto taps) {
        using T = decltype(t);
        constexpr int V = decltype(v)::value, W = decltype(taps)::value;
        hipLaunchKernelGGL((conv1d_step_kernel<T, V, W>),
                           dim3((unsigned)d->tokens, (unsigned)channel_groups(d->channels, V)), dim3(kWave), 0,
                           static_cast<hipStream_t>(stream), a);
    });
    return launched("causal_conv1d_step");
}

}  // extern "C"
