// causal_conv.cu - the short causal convolution along the tokens, one filter per channel, with an activation: forward,
// gradients, and the step of serving.
//
//   z_t = bias + sum_j w_j x_(t - W + 1 + j) over the tokens of one sequence (before its first: the initial state),
//   y_t = act(z_t);   g_t = dy_t act'(z_t),   dx_t = sum_i w_(W - 1 - i) g_(t + i),   dw_j = sum_t g_t x_(t - W + 1 + j).
//
// The bytes are few: x is read and y written once.  A thread takes a vector of four channels and walks along a run of
// tokens, the last W - 1 inputs in registers, so that only the W - 1 inputs before a run are read twice.  24576 x 1536 in bf16, four taps with SiLU: 39 us
// dense (58% of the copy rate), 42 packed (the search for a run's sequence goes beside its first rows); fp32 51 (87%) and 52.  Gradients 94 and 111: filter, sums
// and window fill the registers (128 and 168), so that few rows are on their way.  Runs inside one sequence, nearly all, take a path without
// checks for its borders (without it 59 packed, gradients 129 and 124); 80 registers, six blocks on an SM (without that limit 43 and 48).  Vectors of eight bf16 channels took 177 registers and were slower, rows of eight asked for at once too.
#include <initializer_list>

#include "layer_common.cuh"
#include "layer_internal.h"
#include "vmb_internal.h"

namespace vmb {

namespace {

constexpr int kConvThreads = 128;
constexpr int kConvBatch = 4;  // rows whose values are read before the first is used
template <typename T> constexpr int conv_bwd_blocks_per_sm() { return sizeof(T) == 2 ? 4 : 3; }  // of the gradients: 128 and 168 registers
constexpr int kConvRun = 16;   // rows of a run of the forward at most

// How the threads of a launch lie over the channels: tx vectors side by side, ty runs of tokens, nb blocks over the channels.
struct ConvGrid {
    int tx, ty, nb;
};
ConvGrid conv_grid(int vectors) {
    ConvGrid g;
    g.nb = (vectors + kConvThreads - 1) / kConvThreads;
    g.tx = (vectors + g.nb - 1) / g.nb;
    g.ty = kConvThreads / g.tx;
    return g;
}

struct ConvKernel {
    ConvArgs a;
    ConvGrid g;
    int run;               // tokens of a run
    long long runs;        // of all sequences (dense: runs_per of each; packed: over all rows)
    int runs_per;
    unsigned tile_blocks;  // blocks over the runs; those behind them: states and rows without a sequence
    float* partial;        // gradients: [blocks x ty][W + 1][C]
};

// The inputs before row t (place p in the sequence) that its taps see, oldest first.
template <typename T, int V, int W>
__device__ __forceinline__ void window_before(float (&win)[W > 1 ? W - 1 : 1][V], const T* x, long long x_t, const T* initial, int C, long long p) {
#pragma unroll
    for (int j = 0; j < W - 1; ++j) {
        const long long q = p - (W - 1) + j;
#pragma unroll
        for (int i = 0; i < V; ++i) win[j][i] = 0.0f;
        if (q >= 0) load_vec<T, V>(win[j], x + (q - p) * x_t);
        else if (initial) load_vec<T, V>(win[j], initial + (long long)(W - 1 + q) * C);
    }
}

// z of the row whose input is `cur`, the window moved on by one.
template <int V, int W>
__device__ __forceinline__ void taps(float (&z)[V], float (&win)[W > 1 ? W - 1 : 1][V], const float (&cur)[V], const float (&w)[W][V], const float (&bias)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
        float s = bias[i];
#pragma unroll
        for (int j = 0; j < W - 1; ++j) s = fmaf(w[j][i], win[j][i], s);
        z[i] = fmaf(w[W - 1][i], cur[i], s);
#pragma unroll
        for (int j = 0; j + 2 < W; ++j) win[j][i] = win[j + 1][i];
        if (W > 1) win[W > 1 ? W - 2 : 0][i] = cur[i];
    }
}

template <int V, int W>
__device__ __forceinline__ void load_filter(float (&w)[W][V], float (&bias)[V], const ConvArgs& a, int c) {
    const float* p = a.weight + (long long)c * W;  // [V][W], dense
    if (V * W % 4 == 0 && (reinterpret_cast<uintptr_t>(p) & 15) == 0) {
#pragma unroll
        for (int q = 0; q < V * W / 4; ++q) {
            const float4 f = reinterpret_cast<const float4*>(p)[q];
            const float all[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) w[(4 * q + e) % W][(4 * q + e) / W] = all[e];
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
            for (int j = 0; j < W; ++j) w[j][i] = p[i * W + j];
    }
    if (V % 4 == 0 && (reinterpret_cast<uintptr_t>(a.bias) & 15) == 0) {
#pragma unroll
        for (int q = 0; q < V / 4; ++q) {
            const float4 f = a.bias ? reinterpret_cast<const float4*>(a.bias + c)[q] : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            bias[4 * q % V] = f.x, bias[(4 * q + 1) % V] = f.y, bias[(4 * q + 2) % V] = f.z, bias[(4 * q + 3) % V] = f.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) bias[i] = a.bias ? a.bias[c + i] : 0.0f;
    }
}
template <typename T, int V> __device__ __forceinline__ Vec<T, V> raw_vec(const T* p) { return *reinterpret_cast<const Vec<T, V>*>(p); }
template <typename T, int V> __device__ __forceinline__ void widen(float (&out)[V], const Vec<T, V>& a) {
#pragma unroll
    for (int i = 0; i < V; ++i) out[i] = io<T>::cvt(a.v[i]);
}

// The sequence of a packed row, -1 or B if none has it.
__device__ __forceinline__ int sequence_of(const int* offsets, int B, long long t) {
    int lo = -1, hi = B + 1;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (offsets[mid] <= t) lo = mid;
        else hi = mid;
    }
    return lo;
}

// Walks over the rows of a run and keeps what sequence they are in.
struct Place {
    int b;                  // -1 or B: rows of no sequence
    long long start, end;   // of that sequence, in rows
    __device__ __forceinline__ bool none(int B) const { return b < 0 || b >= B; }
};
__device__ __forceinline__ Place place_in(const int* offsets, int B, long long total, long long row, int b) {
    Place p;
    p.b = b;
    p.start = p.b < 0 ? 0 : min(max((long long)offsets[p.b], 0LL), row);
    p.end = p.b >= B ? total : offsets[p.b + 1];
    if (p.end <= row || p.end > total) p.end = total;
    return p;
}

__device__ __forceinline__ Place place_of(const int* offsets, int B, long long total, long long row) {
    return place_in(offsets, B, total, row, sequence_of(offsets, B, row));
}
// The same for the first rows of a block's runs: by a warp for each while they are few (32 offsets a round), else by a thread.
__device__ __forceinline__ int first_sequence(const ConvArgs& a, const ConvGrid& g, long long first, int run, long long runs) {
    __shared__ int seq[kConvThreads];
    const int w = threadIdx.x >> 5;
    if (g.ty <= 8) {
        for (int r = w; r < g.ty; r += kConvThreads / 32) {
            const int b = last_at_most(a.B, (first + r) * run, [&](int i) { return (long long)a.offsets[i]; });
            if ((threadIdx.x & 31) == 0) seq[r] = b;
        }
    } else if (threadIdx.x < g.ty && first + threadIdx.x < runs) {
        seq[threadIdx.x] = sequence_of(a.offsets, a.B, (first + threadIdx.x) * run);
    }
    __syncthreads();
    const int ly = threadIdx.x / g.tx;
    return ly < g.ty ? seq[ly] : 0;
}

// Final states: the last W - 1 inputs of sequence b, of the initial state where it is shorter.
template <typename T, int V, int W> __device__ __forceinline__ void last_inputs(const ConvArgs& a, int b, int c) {
    long long start = 0, len = a.T;
    const T* x = (const T*)a.x + c;
    if (a.offsets) {
        long long end;
        sequence_span(a.offsets, b, a.total, &start, &end);
        len = end - start;
        x += start * a.x_t;
    } else {
        x += b * a.x_b;
    }
    const long long base = (long long)b * (W - 1) * a.C + c;
#pragma unroll
    for (int j = 0; j < W - 1; ++j) {
        const long long q = len - (W - 1) + j;
        Vec<T, V> v{};
        if (q >= 0) v = *reinterpret_cast<const Vec<T, V>*>(x + q * a.x_t);
        else if (a.initial) v = *reinterpret_cast<const Vec<T, V>*>((const T*)a.initial + base + (long long)(W - 1 + q) * a.C);
        *reinterpret_cast<Vec<T, V>*>((T*)a.final + base + (long long)j * a.C) = v;
    }
}

template <typename T, int V, int W, int ACT, bool kPacked> __global__ void __launch_bounds__(kConvThreads, 6) conv_fwd_kernel(ConvKernel k) {
    const ConvArgs& a = k.a;
    const int lx = threadIdx.x % k.g.tx, ly = threadIdx.x / k.g.tx;
    const int c = (blockIdx.y * k.g.tx + lx) * V;
    pdl_wait();
    pdl_launch_dependents();
    if (blockIdx.x >= k.tile_blocks) {
        const long long b = (long long)(blockIdx.x - k.tile_blocks) * k.g.ty + ly;
        if (b < a.B && c < a.C && ly < k.g.ty) last_inputs<T, V, W>(a, (int)b, c);
        return;
    }
    const long long run = (long long)blockIdx.x * k.g.ty + ly;
    const bool on = c < a.C && ly < k.g.ty && run < k.runs;
    const T *x = (const T*)a.x, *initial = (const T*)a.initial;
    T* y = nullptr;
    long long row = 0, left = 0, before = 0;  // (packed: the row of all; dense: the place in the sequence; rows of x that lie before it)
    if (on) {
        int b = 0;
        if constexpr (kPacked) {
            row = run * k.run;
            left = min((long long)k.run, a.total - row);
            x += row * a.x_t + c;
            y = (T*)a.y + row * a.C + c;
        } else {
            b = (int)(run / k.runs_per);
            row = (run - (long long)b * k.runs_per) * k.run;
            left = min((long long)k.run, a.T - row);
            x += b * a.x_b + row * a.x_t + c;
            y = (T*)a.y + ((long long)b * a.T + row) * a.C + c;
            if (initial) initial += (long long)b * (W - 1) * a.C + c;
        }
        before = row;
    }
    // the first rows and those before them are asked for before the sequence is known
    Vec<T, V> in[kConvBatch], old[W > 1 ? W - 1 : 1];
    auto fetch = [&](long long r) {
#pragma unroll
        for (int u = 0; u < kConvBatch; ++u)
            if (r + u < left) in[u] = raw_vec<T, V>(x + (r + u) * a.x_t);
    };
    fetch(0);
#pragma unroll
    for (int j = 0; j < W - 1; ++j) {
        old[j] = Vec<T, V>{};
        if (on && before - (W - 1) + j >= 0) old[j] = raw_vec<T, V>(x + (long long)(j - (W - 1)) * a.x_t);
    }
    Place at{0, 0, 0};
    long long place = row;  // in the sequence
    if constexpr (kPacked) {
        const int b = first_sequence(a, k.g, (long long)blockIdx.x * k.g.ty, k.run, k.runs);
        if (on) {
            at = place_in(a.offsets, a.B, a.total, row, b);
            place = row - at.start;
            if (initial && !at.none(a.B)) initial += (long long)at.b * (W - 1) * a.C + c;
        }
    }
    if (!on) return;
    float w[W][V], bias[V], win[W > 1 ? W - 1 : 1][V];
    load_filter<V, W>(w, bias, a, c);
#pragma unroll
    for (int j = 0; j < W - 1; ++j) {
        widen<T, V>(win[j], old[j]);
        const long long q = place - (W - 1) + j;
        if (kPacked && at.none(a.B)) continue;
        if (q < 0) {
#pragma unroll
            for (int i = 0; i < V; ++i) win[j][i] = 0.0f;
            if (initial) load_vec<T, V>(win[j], initial + (long long)(W - 1 + q) * a.C);
        }
    }
    if (left == k.run && (!kPacked || (!at.none(a.B) && row + left <= at.end))) {  // a run inside one sequence
#pragma unroll 1
        for (int r = 0; r < k.run; r += kConvBatch) {
            if (r) {
#pragma unroll
                for (int u = 0; u < kConvBatch; ++u) in[u] = raw_vec<T, V>(x + u * a.x_t);
            }
#pragma unroll
            for (int u = 0; u < kConvBatch; ++u) {
                float z[V], cur[V];
                widen<T, V>(cur, in[u]);
                taps<V, W>(z, win, cur, w, bias);
#pragma unroll
                for (int i = 0; i < V; ++i) z[i] = activate<ACT>(z[i]);
                store_vec<T, V>(y + (long long)u * a.C, z);
            }
            x += kConvBatch * a.x_t, y += (long long)kConvBatch * a.C;
        }
        return;
    }
    for (long long r = 0; r < left; r += kConvBatch) {
        if (r) fetch(r);
#pragma unroll
        for (int u = 0; u < kConvBatch; ++u) {
            if (r + u >= left) break;
            if constexpr (kPacked) {
                if (row + r + u == at.end) {
                    at = place_of(a.offsets, a.B, a.total, row + r + u);
                    if (!at.none(a.B))
                        window_before<T, V, W>(win, x + (r + u) * a.x_t, a.x_t, a.initial ? (const T*)a.initial + (long long)at.b * (W - 1) * a.C + c : nullptr, a.C,
                                               row + r + u - at.start);
                }
            }
            float z[V], cur[V];
            widen<T, V>(cur, in[u]);
            taps<V, W>(z, win, cur, w, bias);
#pragma unroll
            for (int i = 0; i < V; ++i) z[i] = kPacked && at.none(a.B) ? 0.0f : activate<ACT>(z[i]);
            store_vec<T, V>(y + (r + u) * a.C, z);
        }
    }
}

// Gradients.  A thread walks its run and the W - 1 rows behind it; `acc` holds the sums of dx of the last W - 1 rows, whose later
// rows are still to come.  Its sums over the tokens go on from run to run and leave one row of partial sums.
template <typename T, int V, int W, int ACT, bool kPacked> __global__ void __launch_bounds__(kConvThreads, conv_bwd_blocks_per_sm<T>()) conv_bwd_kernel(ConvKernel k) {
    const ConvArgs& a = k.a;
    const int lx = threadIdx.x % k.g.tx, ly = threadIdx.x / k.g.tx;
    const int c = (blockIdx.y * k.g.tx + lx) * V;
    pdl_wait();
    pdl_launch_dependents();
    if (c >= a.C || ly >= k.g.ty) return;
    float w[W][V], bias[V], dw[W][V], db[V];
    load_filter<V, W>(w, bias, a, c);
#pragma unroll
    for (int i = 0; i < V; ++i) {
#pragma unroll
        for (int j = 0; j < W; ++j) dw[j][i] = 0.0f;
        db[i] = 0.0f;
    }
    for (long long run = (long long)blockIdx.x * k.g.ty + ly; run < k.runs; run += (long long)k.tile_blocks * k.g.ty) {
        long long row, seq0;  // the run's first row of all, and row - seq0 is its place in x's rows
        const T *x, *dy;
        T* dx;
        long long left, stop;  // rows of the run, and rows until the end of the tensor or sequence
        Place at{0, 0, 0};
        if constexpr (kPacked) {
            row = run * k.run;
            stop = a.total - row;
            x = (const T*)a.x + row * a.x_t + c;
            at = place_of(a.offsets, a.B, a.total, row);
            seq0 = row;
        } else {
            const int b = (int)(run / k.runs_per);
            const long long t = (run - (long long)b * k.runs_per) * k.run;
            stop = a.T - t;
            x = (const T*)a.x + b * a.x_b + t * a.x_t + c;
            at.b = b, at.start = (long long)b * a.T, at.end = at.start + a.T;
            row = at.start + t;
            seq0 = row;
        }
        left = min((long long)k.run, stop);
        dy = (const T*)a.dy + row * a.C + c;
        dx = (T*)a.dx + row * a.C + c;
        float win[W > 1 ? W - 1 : 1][V], acc[W][V];  // acc[j]: row r - j
        auto enter = [&](long long r) {
#pragma unroll
            for (int j = 0; j < W; ++j)
#pragma unroll
                for (int i = 0; i < V; ++i) acc[j][i] = 0.0f;
            if (at.none(a.B)) return;
            const T* initial = a.initial ? (const T*)a.initial + (long long)at.b * (W - 1) * a.C + c : nullptr;
            window_before<T, V, W>(win, x + r * a.x_t, a.x_t, initial, a.C, seq0 + r - at.start);
        };
        // dx of row r, all of whose later rows have been added
        auto leave = [&](long long r, const float (&sum)[V]) {
            if (r < 0 || r >= left || seq0 + r < at.start) return;
            float o[V];
#pragma unroll
            for (int i = 0; i < V; ++i) o[i] = sum[i];
            const long long kept = seq0 + r - at.end + W - 1;  // its place in the final state
            if (a.dfinal && kept >= 0 && kept < W - 1 && !at.none(a.B)) {
                float f[V];
                load_vec<T, V>(f, (const T*)a.dfinal + ((long long)at.b * (W - 1) + kept) * a.C + c);
#pragma unroll
                for (int i = 0; i < V; ++i) o[i] += f[i];
            }
            store_vec<T, V>(dx + r * a.C, o);
        };
        enter(0);
        // a run whose rows, and the W - 1 behind them, are of one sequence: no row of it is among the sequence's last W - 1
        if (left == k.run && !at.none(a.B) && seq0 + left + W - 1 <= at.end) {
            float later[W > 1 ? W - 1 : 1][V];  // g of the last W - 1 rows
            const int xs = (int)a.x_t;
            // g of a row, its input taken into the window
            auto slope_row = [&](float (&g)[V], const Vec<T, V>& rx, const Vec<T, V>& rg, bool sums) {
                float cur[V], z[V];
                widen<T, V>(cur, rx);
                widen<T, V>(g, rg);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    float s = bias[i];
#pragma unroll
                    for (int j = 0; j < W - 1; ++j) s = fmaf(w[j][i], win[j][i], s);
                    z[i] = fmaf(w[W - 1][i], cur[i], s);
                    g[i] *= activate_slope<ACT>(z[i]);
                    if (sums) {
#pragma unroll
                        for (int j = 0; j < W - 1; ++j) dw[j][i] = fmaf(g[i], win[j][i], dw[j][i]);
                        dw[W - 1][i] = fmaf(g[i], cur[i], dw[W - 1][i]);
                        db[i] += g[i];
                    }
#pragma unroll
                    for (int j = 0; j + 2 < W; ++j) win[j][i] = win[j + 1][i];
                    if (W > 1) win[W > 1 ? W - 2 : 0][i] = cur[i];
                }
            };
            // dx of the row W - 1 before the one whose g this is
            auto emit = [&](const float (&g)[V], T* p, bool out) {
                float o[V];
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    o[i] = w[0][i] * g[i];
#pragma unroll
                    for (int j = 0; j < W - 1; ++j) o[i] = fmaf(w[W - 1 - j][i], later[j][i], o[i]);
#pragma unroll
                    for (int j = 0; j + 2 < W; ++j) later[j][i] = later[j + 1][i];
                    if (W > 1) later[W > 1 ? W - 2 : 0][i] = g[i];
                }
                if (out) store_vec<T, V>(p, o);
            };
#pragma unroll
            for (int j = 0; j < W - 1; ++j)
#pragma unroll
                for (int i = 0; i < V; ++i) later[j][i] = 0.0f;
            T* out = dx - (W - 1) * a.C;
#pragma unroll 1
            for (int r = 0; r < k.run; r += kConvBatch) {
                Vec<T, V> rx[kConvBatch], rg[kConvBatch];
#pragma unroll
                for (int u = 0; u < kConvBatch; ++u) rx[u] = raw_vec<T, V>(x + u * xs), rg[u] = raw_vec<T, V>(dy + u * a.C);
#pragma unroll
                for (int u = 0; u < kConvBatch; ++u) {
                    float g[V];
                    slope_row(g, rx[u], rg[u], true);
                    emit(g, out + u * a.C, r + u >= W - 1);
                }
                x += (long long)kConvBatch * xs, dy += (long long)kConvBatch * a.C, out += (long long)kConvBatch * a.C;
            }
#pragma unroll
            for (int u = 0; u < W - 1; ++u) {
                float g[V];
                slope_row(g, raw_vec<T, V>(x + u * xs), raw_vec<T, V>(dy + u * a.C), false);
                emit(g, out + u * a.C, true);
            }
            continue;
        }
        const long long last = min(left + W - 1, stop);
        for (long long r0 = 0; r0 < last; r0 += kConvBatch) {
            Vec<T, V> raw[kConvBatch], rdy[kConvBatch];
#pragma unroll
            for (int u = 0; u < kConvBatch; ++u)
                if (r0 + u < last) raw[u] = raw_vec<T, V>(x + (r0 + u) * a.x_t), rdy[u] = raw_vec<T, V>(dy + (r0 + u) * a.C);
#pragma unroll
            for (int u = 0; u < kConvBatch; ++u) {
                const long long r = r0 + u;
                if (r >= last) break;
                if constexpr (kPacked) {
                    if (seq0 + r == at.end) {  // the last rows of a sequence have no later ones
#pragma unroll
                        for (int j = W - 1; j >= 1; --j) leave(r - j, acc[j - 1]);
                        at = place_of(a.offsets, a.B, a.total, seq0 + r);
                        enter(r);
                    }
                }
                if (kPacked && at.none(a.B)) {
                    if (r < left) {
                        const float zero[V] = {};
                        store_vec<T, V>(dx + r * a.C, zero);
                    }
                    continue;
                }
                float z[V], old[W > 1 ? W - 1 : 1][V], g[V], in[V], gy[V];
                widen<T, V>(in, raw[u]);
                widen<T, V>(gy, rdy[u]);
#pragma unroll
                for (int j = 0; j < W - 1; ++j)
#pragma unroll
                    for (int i = 0; i < V; ++i) old[j][i] = win[j][i];
                taps<V, W>(z, win, in, w, bias);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    g[i] = gy[i] * activate_slope<ACT>(z[i]);
                    if (r < left) {
#pragma unroll
                        for (int j = 0; j < W - 1; ++j) dw[j][i] = fmaf(g[i], old[j][i], dw[j][i]);
                        dw[W - 1][i] = fmaf(g[i], in[i], dw[W - 1][i]);
                        db[i] += g[i];
                    }
#pragma unroll
                    for (int j = W - 1; j >= 1; --j) acc[j][i] = fmaf(w[W - 1 - j][i], g[i], acc[j - 1][i]);
                    acc[0][i] = w[W - 1][i] * g[i];
                }
                leave(r - (W - 1), acc[W - 1]);
            }
        }
        if (last == stop && !at.none(a.B)) {  // the last rows of all: nothing behind them
#pragma unroll
            for (int j = W - 1; j >= 1; --j) leave(last - j, acc[j - 1]);
        }
    }
    float* p = k.partial + ((long long)blockIdx.x * k.g.ty + ly) * (W + 1) * a.C + c;
#pragma unroll
    for (int i = 0; i < V; ++i) {
#pragma unroll
        for (int j = 0; j < W; ++j) p[(long long)j * a.C + i] = dw[j][i];
        p[(long long)W * a.C + i] = db[i];
    }
}

// The gradient of the initial state: row i meets the first tokens t <= i with tap i - t; of a sequence shorter than W - 1 tokens it
// is in the final state too.
template <typename T, int W, int ACT> __global__ void __launch_bounds__(128) conv_dinitial_kernel(ConvArgs a) {
    pdl_wait();
    pdl_launch_dependents();
    const long long item = (long long)blockIdx.x * 128 + threadIdx.x;
    if (item >= (long long)a.B * a.C) return;
    const int b = (int)(item / a.C), c = (int)(item % a.C);
    long long start = (long long)b * a.T, len = a.T;
    const T* x = (const T*)a.x + c;
    if (a.offsets) {
        long long end;
        sequence_span(a.offsets, b, a.total, &start, &end);
        len = end - start;
        x += start * a.x_t;
    } else {
        x += b * a.x_b;
    }
    float w[W][1], bias[1], win[W > 1 ? W - 1 : 1][1], out[W];
    load_filter<1, W>(w, bias, a, c);
    const long long base = (long long)b * (W - 1) * a.C + c;
    window_before<T, 1, W>(win, x, a.x_t, a.initial ? (const T*)a.initial + base : nullptr, a.C, 0);
#pragma unroll
    for (int i = 0; i < W; ++i) out[i] = 0.0f;
#pragma unroll
    for (int t = 0; t < W - 1; ++t) {
        if (t >= len) break;
        float z[1], cur[1] = {io<T>::cvt(x[t * a.x_t])};
        taps<1, W>(z, win, cur, w, bias);
        const float g = io<T>::cvt(((const T*)a.dy)[(start + t) * a.C + c]) * activate_slope<ACT>(z[0]);
#pragma unroll
        for (int i = 0; i < W - 1; ++i)
            if (i >= t) out[i] = fmaf(w[i - t][0], g, out[i]);
    }
    for (int i = 0; i < W - 1; ++i) {
        if (a.dfinal && i >= len) out[i] += io<T>::cvt(((const T*)a.dfinal)[base + (long long)(i - len) * a.C]);
        ((T*)a.dinitial)[base + (long long)i * a.C] = io<T>::to(out[i]);
    }
}

// Sums of columns: a warp's lanes are columns, the warps of a block take the rows in turn, their sums are joined in order.
__global__ void __launch_bounds__(512) column_sums_kernel(const float* p, int rows, long long cols, int C, int taps, float* out, float* rest, int n_rest, float* more) {
    __shared__ float part[16][33];
    pdl_wait();
    pdl_launch_dependents();
    const int lane = threadIdx.x & 31, wp = threadIdx.x >> 5;
    const long long col = (long long)blockIdx.x * 32 + lane;
    float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (col < cols) {
        int r = wp;
        for (; r + 48 < rows; r += 64)
#pragma unroll
            for (int u = 0; u < 4; ++u) s[u] += p[(long long)(r + 16 * u) * cols + col];
        for (; r < rows; r += 16) s[0] += p[(long long)r * cols + col];
    }
    part[wp][lane] = (s[0] + s[1]) + (s[2] + s[3]);
    __syncthreads();
    if (wp == 0 && col < cols) {
        float v = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) v += part[i][lane];
        const long long main = (long long)taps * C;
        if (col >= main) {
            const long long at = col - main;
            if (at < n_rest) {
                if (rest) rest[at] = v;
            } else if (more) {
                more[at - n_rest] = v;
            }
        } else if (out) {
            out[taps == 1 ? col : (col % C) * taps + col / C] = v;
        }
    }
}

// A few tokens of every row from the inputs kept in its slot, which move on.
template <typename T, int V, int W, int ACT> __global__ void __launch_bounds__(kConvThreads) conv_step_kernel(ConvKernel k) {
    const ConvArgs& a = k.a;
    const int lx = threadIdx.x % k.g.tx, ly = threadIdx.x / k.g.tx;
    const int c = (blockIdx.y * k.g.tx + lx) * V;
    const long long b = (long long)blockIdx.x * k.g.ty + ly;
    pdl_wait();
    pdl_launch_dependents();
    if (c >= a.C || ly >= k.g.ty || b >= a.B) return;
    const long long slot = a.slots ? a.slots[b] : b;
    T* y = (T*)a.y + b * a.T * a.C + c;
    if (slot < 0 || slot >= a.pool) {
        const float zero[V] = {};
        for (int t = 0; t < a.T; ++t) store_vec<T, V>(y + (long long)t * a.C, zero);
        return;
    }
    float w[W][V], bias[V], win[W > 1 ? W - 1 : 1][V], in[V], z[V];
    load_filter<V, W>(w, bias, a, c);
    T* state = (T*)a.state + slot * (W - 1) * a.C + c;
#pragma unroll
    for (int j = 0; j < W - 1; ++j) load_vec<T, V>(win[j], state + (long long)j * a.C);
    const T* x = (const T*)a.x + b * a.x_b + c;
    for (int t = 0; t < a.T; ++t) {
        load_vec<T, V>(in, x + t * a.x_t);
        taps<V, W>(z, win, in, w, bias);
#pragma unroll
        for (int i = 0; i < V; ++i) z[i] = activate<ACT>(z[i]);
        store_vec<T, V>(y + (long long)t * a.C, z);
    }
#pragma unroll
    for (int j = 0; j < W - 1; ++j) store_vec<T, V>(state + (long long)j * a.C, win[j]);
}

enum ConvWhat { kFwd, kBwd, kStep, kDinitial };

template <typename T, int V, int W, int ACT> const void* conv_fn(ConvWhat what, bool packed) {
    if (what == kFwd) return packed ? (const void*)conv_fwd_kernel<T, V, W, ACT, true> : (const void*)conv_fwd_kernel<T, V, W, ACT, false>;
    if (what == kBwd) return packed ? (const void*)conv_bwd_kernel<T, V, W, ACT, true> : (const void*)conv_bwd_kernel<T, V, W, ACT, false>;
    if (what == kStep) return (const void*)conv_step_kernel<T, V, W, ACT>;
    return (const void*)conv_dinitial_kernel<T, W, ACT>;
}
template <typename T, int V> const void* conv_fn(ConvWhat what, int W, vmb_act act, bool packed) {
    if (act == VMB_ACT_SILU)
        return W == 1   ? conv_fn<T, V, 1, VMB_ACT_SILU>(what, packed)
               : W == 2 ? conv_fn<T, V, 2, VMB_ACT_SILU>(what, packed)
               : W == 3 ? conv_fn<T, V, 3, VMB_ACT_SILU>(what, packed)
                        : conv_fn<T, V, 4, VMB_ACT_SILU>(what, packed);
    return W == 1   ? conv_fn<T, V, 1, VMB_ACT_NONE>(what, packed)
           : W == 2 ? conv_fn<T, V, 2, VMB_ACT_NONE>(what, packed)
           : W == 3 ? conv_fn<T, V, 3, VMB_ACT_NONE>(what, packed)
                    : conv_fn<T, V, 4, VMB_ACT_NONE>(what, packed);
}

// Vectors of four channels, or single channels where rows or pointers do not allow them.
bool conv_vectors(const ConvArgs& a) {
    const int V = 4;
    if (a.C % V || a.x_t % V || (!a.offsets && a.B > 1 && a.x_b % V)) return false;
    for (const void* p : {a.x, (const void*)a.y, a.initial, (const void*)a.final, a.dy, a.dfinal, (const void*)a.dx, (const void*)a.state})
        if (reinterpret_cast<uintptr_t>(p) & 15) return false;
    return true;
}
const void* conv_kernel(const ConvArgs& a, ConvWhat what, bool vec) {
    if (a.dtype == VMB_BF16)
        return vec ? conv_fn<__nv_bfloat16, 4>(what, a.W, a.act, a.offsets != nullptr) : conv_fn<__nv_bfloat16, 1>(what, a.W, a.act, a.offsets != nullptr);
    return vec ? conv_fn<float, 4>(what, a.W, a.act, a.offsets != nullptr) : conv_fn<float, 1>(what, a.W, a.act, a.offsets != nullptr);
}

// Runs of 16 tokens (the W - 1 inputs before a run then add at most a fifth to what the L1 and L2 caches deliver), of four
// where the launch would not fill the SMs.
void conv_runs(ConvKernel& k, int most) {
    const ConvArgs& a = k.a;
    const long long fill = 4LL * device_sm_count() * 512 / k.g.nb / k.g.tx;
    k.run = most;
    while (k.run > 4 && a.total / k.run < fill) k.run /= 2;
    k.runs_per = (a.T + k.run - 1) / k.run;
    k.runs = a.offsets ? (a.total + k.run - 1) / k.run : (long long)a.B * k.runs_per;
}

unsigned conv_bwd_blocks(const ConvKernel& k) {
    const long long want = (k.runs + k.g.ty - 1) / k.g.ty;
    long long most = (long long)device_sm_count() * (k.a.dtype == VMB_BF16 ? conv_bwd_blocks_per_sm<__nv_bfloat16>() : conv_bwd_blocks_per_sm<float>()) / k.g.nb;
    if (most < 1) most = 1;
    return (unsigned)(want < 1 ? 1 : want < most ? want : most);
}

}  // namespace

vmb_status launch_column_sums(const float* p, int rows, long long cols, int C, int taps, float* out, float* rest, int n_rest, float* more,
                              cudaStream_t stream) {
    void* args[] = {&p, &rows, &cols, &C, &taps, &out, &rest, &n_rest, &more};
    return launch_kernel((const void*)column_sums_kernel, dim3((unsigned)((cols + 31) / 32)), dim3(512), 0, args, stream) == cudaSuccess
               ? VMB_OK : VMB_ERR_CUDA;
}

// One row of partial sums for each run of threads of the gradients' launch, whichever vectors it takes.
size_t conv_workspace_bytes(int, int, long long, bool, int C, int W, vmb_dtype dtype) {
    size_t most = 0;
    for (int V : {1, 4}) {
        const ConvGrid g = conv_grid((C + V - 1) / V);
        long long blocks = (long long)device_sm_count() * 4 / g.nb;
        if (blocks < 1) blocks = 1;
        const size_t n = (size_t)blocks * g.ty * (W + 1) * C * 4;
        if (n > most) most = n;
    }
    return align_up(most, 256) + 256;
}

vmb_status launch_conv_fwd(const ConvArgs& a, cudaStream_t stream) {
    const bool vec = conv_vectors(a);
    const int V = !vec ? 1 : 4;
    ConvKernel k{a, conv_grid((a.C + V - 1) / V)};
    conv_runs(k, kConvRun);
    k.tile_blocks = (unsigned)((k.runs + k.g.ty - 1) / k.g.ty);
    k.partial = nullptr;
    const unsigned states = a.final && a.W > 1 ? (unsigned)(((long long)a.B + k.g.ty - 1) / k.g.ty) : 0u;
    if (k.tile_blocks + states == 0) return VMB_OK;
    void* args[] = {&k};
    return launch_kernel(conv_kernel(a, kFwd, vec), dim3(k.tile_blocks + states, (unsigned)k.g.nb), dim3(kConvThreads), 0, args, stream) == cudaSuccess
               ? VMB_OK : VMB_ERR_CUDA;
}

vmb_status launch_conv_bwd(const ConvArgs& a, cudaStream_t stream) {
    const bool vec = conv_vectors(a);
    const int V = !vec ? 1 : 4;
    ConvKernel k{a, conv_grid((a.C + V - 1) / V)};
    conv_runs(k, 32);
    k.tile_blocks = conv_bwd_blocks(k);
    const int rows = (int)k.tile_blocks * k.g.ty;
    const size_t need = (size_t)rows * (a.W + 1) * a.C * 4;
    if (a.ws_bytes < need + 256) return VMB_ERR_WORKSPACE;
    k.partial = (float*)((char*)a.ws + 256);
    void* args[] = {&k};
    if (launch_kernel(conv_kernel(a, kBwd, vec), dim3(k.tile_blocks, (unsigned)k.g.nb), dim3(kConvThreads), 0, args, stream) != cudaSuccess)
        return VMB_ERR_CUDA;
    if (a.dinitial && a.W > 1 && a.B > 0) {
        ConvArgs g = a;
        void* dargs[] = {&g};
        if (launch_kernel(conv_kernel(a, kDinitial, false), dim3((unsigned)(((long long)a.B * a.C + 127) / 128)), dim3(128), 0, dargs, stream) != cudaSuccess)
            return VMB_ERR_CUDA;
    }
    // partial rows hold [W + 1][C]: the taps, then the bias
    return launch_column_sums(k.partial, rows, (long long)(a.W + 1) * a.C, a.C, a.W, a.dweight, a.dbias, a.C, nullptr, stream);
}

vmb_status launch_conv_step(const ConvArgs& a, cudaStream_t stream) {
    const bool vec = conv_vectors(a);
    const int V = !vec ? 1 : 4;
    ConvKernel k{a, conv_grid((a.C + V - 1) / V)};
    void* args[] = {&k};
    return launch_kernel(conv_kernel(a, kStep, vec), dim3((unsigned)(((long long)a.B + k.g.ty - 1) / k.g.ty), (unsigned)k.g.nb), dim3(kConvThreads), 0, args,
                         stream) == cudaSuccess ? VMB_OK : VMB_ERR_CUDA;
}

}  // namespace vmb
