// token_scan_grad.cu - gradients of the selective scan over tokens.
//
// With g_t = dy_t silu(z_t) (dy_t without a gate), a_t = exp(dt_t A) and the adjoint of the state
//   lam_t = C_t g_t + a_(t+1) lam_(t+1):
//   dx = dt (lam . B) + D g,   ddt = x (lam . B) + sum_n A a h_(t-1) lam,   ddelta = ddt softplus'(delta + bias),
//   dB = sum_channels lam dt x,   dC = sum_channels g h_t,   dz = dy (C . h + D x) silu'(z),
//   dA = sum_tokens dt a h_(t-1) lam,   dD = sum g x,   dbias = sum ddelta.
//
// The states are formed again from those that the forward kept before every 16 tokens.  A sequence is cut into segments: a first
// launch leaves what each segment's tokens give to the adjoint before it (a sum without a recurrence: the product of the
// decays up to a token is the exponential of A times the sum of the step sizes), and a segment of the second launch starts from
// the joined sums of those behind it.  Three exponentials for each state, and the sums over the channels (a thread's two at once, a warp's
// eight pairs by shuffles, a CTA's four warps through shared memory, the tiles by a third launch, in a fixed order) are what bounds it.
//
// 38 sequences of 2048 tokens of 1024 channels and 16 states with a gate: 2157 us in bf16, 2239 in fp32, 212 instructions for a token of 16 channels at 0.47 a clock and
// scheduler.  With one channel a thread, eight tokens at a time and states kept every 64 tokens, so formed three times, 137 for eight channels: 2689
// and 2940.  Decays formed again instead of kept, for three CTAs on an SM instead of two: 2191 and 2349.
#include "token_scan.cuh"

namespace vmb {

namespace {

// ------------------------------------------------------------ the adjoint of each segment alone

template <typename T, int NP> struct AdjointSmem {
    static constexpr int array = 32 * scan_pitch<T>(), bytes = 3 * array + 32 * NP * 4;
};

template <typename T, int NP> __global__ void __launch_bounds__(kScanThreads, 2) token_scan_adjoint_kernel(ScanKernel k) {
    constexpr int SPL = NP / 4, TOK = 32;
    using L = AdjointSmem<T, NP>;
    extern __shared__ __align__(16) char smem[];
    pdl_wait();
    pdl_launch_dependents();
    const TokenScanArgs& a = k.a;
    const int tile = blockIdx.x % k.tiles, tid = threadIdx.x, q = tid & 3, ch = tid >> 2, c0 = tile * kScanCh, d = c0 + ch, n0 = q * SPL;
    const int cols = min(kScanCh, a.D - c0);
    const long long slot = blockIdx.x / k.tiles;
    const ScanSegment g = scan_segment(k, slot);
    if (!g.live || g.s == 0) return;  // (nothing lies before the first segment)
    float* rows = (float*)(smem + 3 * L::array);
    const bool on = d < a.D;
    Pairs<SPL> A2, acc;
    A2.zero(), acc.zero();
    if (on) {
        A2.load_some(a.A + (long long)d * a.N + n0, n0, a.N);
#pragma unroll
        for (int p = 0; p < Pairs<SPL>::P; ++p) A2.v[p] = __fmul2_rn(A2.v[p], twice(kLog2e));
    }
    const float bias = on && a.bias ? a.bias[d] : 0.0f;
    const T *raw = scan_row<T>(a.delta, a, g, a.d_b, a.d_t) + c0, *dy = (const T*)a.dy + g.first * a.D + c0;
    const T *z = a.z ? scan_row<T>(a.z, a, g, a.z_b, a.z_t) + c0 : nullptr, *Cm = scan_row<T>(a.Cm, a, g, a.C_b, a.C_t);
    float sum = 0.0f;  // of the channel's step sizes
    for (int t0 = 0; t0 < g.len; t0 += TOK) {
        const int left = g.len - t0;
        if (t0) __syncthreads();
        stage_rows<T>(smem, dy + (long long)t0 * a.D, a.D, TOK, left, cols, k.vec);
        stage_rows<T>(smem + L::array, raw + t0 * a.d_t, a.d_t, TOK, left, cols, k.vec);
        if (z) stage_rows<T>(smem + 2 * L::array, z + t0 * a.z_t, a.z_t, TOK, left, cols, k.vec);
        stage_states<T, NP, TOK>(rows, Cm + t0 * a.C_t, a.C_t, a.N, left);
        cp_async_commit();
        cp_async_wait<0>();
        __syncthreads();
#pragma unroll 2
        for (int t = 0; t < TOK; t += 4) {
            float gy = staged<T>(smem, t + q, ch), dt = staged<T>(smem + L::array, t + q, ch) + bias;
            if (z) gy *= activate<VMB_ACT_SILU>(staged<T>(smem + 2 * L::array, t + q, ch));
            if (a.softplus) dt = softplus(dt);
            if (t + q >= left) dt = 0.0f;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const float gu = from_lane(gy, u);
                sum += from_lane(dt, u);
                Pairs<SPL> C, e;
                C.load(rows + (t + u) * NP + n0);
                decays(e, A2, sum);
#pragma unroll
                for (int p = 0; p < Pairs<SPL>::P; ++p) acc.v[p] = __ffma2_rn(e.v[p], __fmul2_rn(C.v[p], twice(gu)), acc.v[p]);
            }
        }
    }
    if (!on) return;
    const long long at = slot * a.D + d;
    acc.store(k.local + at * NP + n0);
    if (q == 0) k.decay[at] = sum;
}

// ------------------------------------------------------------ the gradients of a segment

// Four lanes hold the states of two channels side by side, so that a warp has 16 channels and the sums over the channels begin in a thread.
// A lane reads and prepares one token of every four, for both.  Chunks of 16 tokens, from the last to the first: from the saved state the
// states before each four tokens; then, for four tokens at a time from the last, their states again, kept with their decays in
// registers, and the adjoint back through them.
constexpr int kGradThreads = 128, kChunk = kScanSaved, kQuads = kChunk / 4, kGradWarps = kGradThreads / 32;
// Shared memory: B and C of two chunks, each warp's sums over its channels of two chunks, the states before each four tokens, and what a lane has
// prepared of its tokens (x, step size, its slope, dy, z), all in fp32.
template <int NP> struct GradSmem {
    static constexpr int bc = kChunk * 2 * NP, red = kGradWarps * kChunk * 32, starts = kGradThreads * NP / 2, own = kQuads * kGradThreads * 2;
    static constexpr int floats = 2 * bc + 2 * red + kQuads * starts + 5 * own, bytes = floats * 4;
};

// The sums over the eight channels of a warp of 2 SPL values for each of the four lanes of a channel; lane l is left with that of
// (dB or dC, state) as bc_lane gives it.
template <int SPL> __device__ __forceinline__ float channel_sums(float (&v)[2 * SPL]) {
    const int lane = threadIdx.x & 31;
    int n = 2 * SPL;
#pragma unroll
    for (int d = 16; d >= 4; d >>= 1) {
        const bool hi = lane & d;
        if (n > 1) {
            n /= 2;
#pragma unroll
            for (int i = 0; i < SPL; ++i) {
                if (i >= n) break;
                const float keep = hi ? v[i + n] : v[i], send = hi ? v[i] : v[i + n];
                v[i] = keep + __shfl_xor_sync(0xffffffffu, send, d);
            }
        } else {
            v[0] += __shfl_xor_sync(0xffffffffu, v[0], d);
        }
    }
    return v[0];
}
template <int SPL> __device__ __forceinline__ int bc_lane(bool is_c, int n) {
    const int q = n / SPL, i = (is_c ? SPL : 0) + n % SPL;  // of 2 SPL values, the highest bit on lane bit 16
    if (SPL == 4) return q + ((i >> 2) & 1) * 16 + ((i >> 1) & 1) * 8 + (i & 1) * 4;
    if (SPL == 2) return q + ((i >> 1) & 1) * 16 + (i & 1) * 8;
    return q + (i & 1) * 16;
}

// A lane's two channels of a token, as they are stored: kept so until they are used, which may be long after they were asked for.
template <typename T> struct Words;
template <> struct Words<float> {
    uint2 w;
    __device__ __forceinline__ float a() const { return __uint_as_float(w.x); }
    __device__ __forceinline__ float b() const { return __uint_as_float(w.y); }
    __device__ __forceinline__ void load(const float* p, bool pair, int next) {
        if (pair) w = *reinterpret_cast<const uint2*>(p);
        else w = make_uint2(__float_as_uint(p[0]), __float_as_uint(p[next]));
    }
};
template <> struct Words<__nv_bfloat16> {
    uint32_t w;
    __device__ __forceinline__ float a() const { return __uint_as_float(w << 16); }
    __device__ __forceinline__ float b() const { return __uint_as_float(w & 0xffff0000u); }
    __device__ __forceinline__ void load(const __nv_bfloat16* p, bool pair, int next) {
        if (pair) w = *reinterpret_cast<const uint32_t*>(p);
        else w = __bfloat16_as_ushort(p[0]) | (uint32_t)__bfloat16_as_ushort(p[next]) << 16;
    }
};
template <typename T> struct alignas(2 * sizeof(T)) Two { T a, b; };
template <typename T> __device__ __forceinline__ void store_two(T* p, float a, float b, bool pair, bool both) {
    if (pair) {
        *reinterpret_cast<Two<T>*>(p) = Two<T>{io<T>::to(a), io<T>::to(b)};
    } else {
        p[0] = io<T>::to(a);
        if (both) p[1] = io<T>::to(b);
    }
}

template <typename T, int NP> __global__ void __launch_bounds__(kGradThreads, 2) token_scan_grad_kernel(ScanKernel k) {
    constexpr int SPL = NP / 4, P = Pairs<SPL>::P, kEach = kChunk * 2 * NP / kGradThreads, kRows = kGradThreads / (2 * NP);
    using L = GradSmem<NP>;
    extern __shared__ __align__(16) float shared[];
    float *bcs = shared, *red = bcs + 2 * L::bc, *starts = red + 2 * L::red;
    float2* own = reinterpret_cast<float2*>(starts + kQuads * L::starts) + threadIdx.x;
    const auto kept = [&](int what, int j) -> float2& { return own[(what * kQuads + j) * kGradThreads]; };
    enum { kX, kDt, kSlope, kDy, kZ };
    pdl_wait();
    pdl_launch_dependents();
    const TokenScanArgs& a = k.a;
    const int tile = blockIdx.x % k.tiles, tid = threadIdx.x, lane = tid & 31, w = tid >> 5, q = tid & 3;
    const int c0 = tile * kScanCh, d = c0 + w * 16 + (lane >> 2) * 2, n0 = q * SPL;
    const long long slot = blockIdx.x / k.tiles;
    if (slot >= k.slots) {  // rows before the first and behind the last sequence (B's and C's are cleared by the sums over the tiles)
        const int cols = min(kScanCh, a.D - c0);
        const long long lo = min(max((long long)a.offsets[0], 0LL), a.total), hi = min(max((long long)a.offsets[a.B], lo), a.total);
        for (long long r = slot - k.slots; r < a.total - (hi - lo); r += kClearBlocks)
            for (int c = tid; c < cols; c += kGradThreads) {
                const long long at = (r < lo ? r : r + hi - lo) * a.D + c0 + c;
                ((T*)a.dx)[at] = ((T*)a.ddelta)[at] = io<T>::to(0.0f);
                if (a.z) ((T*)a.dz)[at] = io<T>::to(0.0f);
            }
        return;
    }
    const ScanSegment g = scan_segment(k, slot);
    const bool on = d < a.D, both = d + 1 < a.D, pair = k.pair;
    const int dd = on ? d : k.pair ? a.D - 2 : a.D - 1, next = both ? 1 : 0;  // (lanes behind the last channel keep their warp's shuffles whole)
    const long long DN = (long long)a.D * a.N;
    float* params = k.params + slot * (DN + 2 * a.D);
    Pairs<SPL> A2[2], lam[2], dA[2];
    float dskip[2] = {0.0f, 0.0f}, dbias[2] = {0.0f, 0.0f};
#pragma unroll
    for (int c = 0; c < 2; ++c) A2[c].zero(), lam[c].zero(), dA[c].zero();
    if (g.live) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int dc = dd + c * next;
            A2[c].load_some(a.A + (long long)dc * a.N + n0, n0, a.N);
#pragma unroll
            for (int p = 0; p < P; ++p) A2[c].v[p] = __fmul2_rn(A2[c].v[p], twice(kLog2e));
            if (!(c ? both : on)) continue;
            if (a.dfinal) lam[c].load_some(a.dfinal + (long long)g.b * DN + (long long)dc * a.N + n0, n0, a.N);
#pragma unroll 4
            for (int s = g.segs - 1; s > g.s; --s) {
                const long long at = (g.place + s) * a.D + dc;
                Pairs<SPL> l, e;
                l.load(k.local + at * NP + n0);
                decays(e, A2[c], k.decay[at]);
#pragma unroll
                for (int p = 0; p < P; ++p) lam[c].v[p] = __ffma2_rn(e.v[p], lam[c].v[p], l.v[p]);
            }
        }
        float bias[2], skip[2];
#pragma unroll
        for (int c = 0; c < 2; ++c) bias[c] = a.bias ? a.bias[dd + c * next] : 0.0f, skip[c] = a.skip ? a.skip[dd + c * next] : 0.0f;
        const T *x = scan_row<T>(a.x, a, g, a.x_b, a.x_t) + dd, *raw = scan_row<T>(a.delta, a, g, a.d_b, a.d_t) + dd;
        const T *z = a.z ? scan_row<T>(a.z, a, g, a.z_b, a.z_t) + dd : nullptr, *dy = (const T*)a.dy + g.first * a.D + dd;
        const long long out0 = g.first * a.D + d;
        const int bn = tid % (2 * NP), brow = tid / (2 * NP);
        const bool bin = bn < NP ? bn < a.N : bn - NP < a.N;
        const long long bs = bn < NP ? a.B_t : a.C_t;
        const T* bc = bn < NP ? scan_row<T>(a.Bm, a, g, a.B_b, a.B_t) + bn : scan_row<T>(a.Cm, a, g, a.C_b, a.C_t) + (bn - NP);
        const float* saved = a.saved + (g.chunk + (long long)g.s * (k.seg / kChunk)) * DN + (long long)dd * a.N + n0;
        const int chunks = (g.len + kChunk - 1) / kChunk;

        Words<T> rx[kQuads], rd[kQuads], rg[kQuads], rz[kQuads];
        T rbc[kEach];
        Pairs<SPL> h[2];
        auto load = [&](int c) {  // (rows behind the last: the last again)
#pragma unroll
            for (int j = 0; j < kQuads; ++j) {
                const long long t = min(c * kChunk + 4 * j + q, g.len - 1);
                rx[j].load(x + t * a.x_t, pair, next), rd[j].load(raw + t * a.d_t, pair, next), rg[j].load(dy + t * a.D, pair, next);
                if (z) rz[j].load(z + t * a.z_t, pair, next);
            }
#pragma unroll
            for (int j = 0; j < kEach; ++j) {
                const int t = c * kChunk + brow + j * kRows;
                rbc[j] = bin && t < g.len ? bc[t * bs] : io<T>::to(0.0f);
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const float* from = saved + c * DN + (long long)(u * next) * a.N;
                if (a.N == NP) h[u].load(from);  // (16-byte aligned)
                else h[u].load_some(from, n0, a.N);
            }
        };
        auto store_bc = [&](float* s) {
#pragma unroll
            for (int j = 0; j < kEach; ++j) s[tid + j * kGradThreads] = io<T>::cvt(rbc[j]);
        };
        if (chunks > 0) {
            load(chunks - 1);
            store_bc(bcs + ((chunks - 1) & 1) * L::bc);
        }
        __syncthreads();
        for (int c = chunks - 1; c >= 0; --c) {
            const int t0 = c * kChunk, left = g.len - t0;
            const float* rows = bcs + (c & 1) * L::bc + n0;
            float* mine = red + (c & 1) * L::red + w * (kChunk * 32) + lane;
            // what this lane has of its tokens
#pragma unroll
            for (int j = 0; j < kQuads; ++j) {
                const bool in = on && 4 * j + q < left, in1 = in && both;  // (nothing else may reach the sums over the channels)
                const auto wide = [&](const Words<T>& v) { return make_float2(in ? v.a() : 0.0f, in1 ? v.b() : 0.0f); };
                float v[2] = {rd[j].a() + bias[0], rd[j].b() + bias[1]}, slope[2] = {1.0f, 1.0f};
                if (a.softplus) {
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const float e = softplus_e(v[u]);
                        slope[u] = softplus_grad_from_e(v[u], e);
                        v[u] = softplus_from_e(v[u], e);
                    }
                }
                kept(kX, j) = wide(rx[j]), kept(kDy, j) = wide(rg[j]);
                kept(kDt, j) = make_float2(in ? v[0] : 0.0f, in1 ? v[1] : 0.0f);
                kept(kSlope, j) = make_float2(slope[0], slope[1]);
                if (z) kept(kZ, j) = wide(rz[j]);
            }
            // the states before each four tokens
#pragma unroll 1
            for (int j = 0; j < kQuads; ++j) {
                float* to = starts + j * L::starts + tid * 2 * SPL;
                h[0].store(to), h[1].store(to + SPL);
                if (j == kQuads - 1) break;
                const float2 dt = kept(kDt, j), dtx = __fmul2_rn(dt, kept(kX, j));
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    Pairs<SPL> B, e0, e1;
                    B.load(rows + (4 * j + i) * 2 * NP);
                    decays(e0, A2[0], from_lane(dt.x, i));
                    decays(e1, A2[1], from_lane(dt.y, i));
                    const float2 u0 = twice(from_lane(dtx.x, i)), u1 = twice(from_lane(dtx.y, i));
#pragma unroll
                    for (int p = 0; p < P; ++p) {
                        h[0].v[p] = __ffma2_rn(e0.v[p], h[0].v[p], __fmul2_rn(u0, B.v[p]));
                        h[1].v[p] = __ffma2_rn(e1.v[p], h[1].v[p], __fmul2_rn(u1, B.v[p]));
                    }
                }
            }
            if (c > 0) load(c - 1);
#pragma unroll 1
            for (int j = kQuads - 1; j >= 0; --j) {
                if (4 * j >= left) continue;  // (the same for the whole CTA)
                const float2 x2 = kept(kX, j), dt2 = kept(kDt, j), dy2 = kept(kDy, j);
                const float xv[2] = {x2.x, x2.y}, dt[2] = {dt2.x, dt2.y}, dyv[2] = {dy2.x, dy2.y}, dtx[2] = {dt2.x * x2.x, dt2.y * x2.y};
                float gy[2] = {dy2.x, dy2.y}, gs[2] = {0.0f, 0.0f};
                if (z) {
                    const float2 z2 = kept(kZ, j);
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const float zv = u ? z2.y : z2.x, s = logistic(zv);
                        gs[u] = s * fmaf(zv, 1.0f - s, 1.0f);
                        gy[u] *= zv * s;
                    }
                }
                Pairs<SPL> e[4][2], before[4][2], now[2];
                now[0].load(starts + j * L::starts + tid * 2 * SPL), now[1].load(starts + j * L::starts + tid * 2 * SPL + SPL);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    Pairs<SPL> B;
                    B.load(rows + (4 * j + i) * 2 * NP);
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        decays(e[i][u], A2[u], from_lane(dt[u], i));
                        const float2 in = twice(from_lane(dtx[u], i));
                        before[i][u] = now[u];
#pragma unroll
                        for (int p = 0; p < P; ++p) now[u].v[p] = __ffma2_rn(e[i][u].v[p], now[u].v[p], __fmul2_rn(in, B.v[p]));
                    }
                }
                float into[2][4], back[2][4], out[2][4];
#pragma unroll
                for (int i = 3; i >= 0; --i) {
                    Pairs<SPL> B, C;
                    B.load(rows + (4 * j + i) * 2 * NP);
                    C.load(rows + (4 * j + i) * 2 * NP + NP);
                    float2 gb[P], gc[P];
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const float2 gu = twice(from_lane(gy[u], i)), dtu = twice(from_lane(dt[u], i)), dxu = twice(from_lane(dtx[u], i));
                        float2 s1, s2, s3;
#pragma unroll
                        for (int p = 0; p < P; ++p) {
                            s3 = p ? __ffma2_rn(C.v[p], now[u].v[p], s3) : __fmul2_rn(C.v[p], now[u].v[p]);
                            lam[u].v[p] = __ffma2_rn(C.v[p], gu, lam[u].v[p]);
                            gc[p] = u ? __ffma2_rn(gu, now[u].v[p], gc[p]) : __fmul2_rn(gu, now[u].v[p]);
                            gb[p] = u ? __ffma2_rn(lam[u].v[p], dxu, gb[p]) : __fmul2_rn(lam[u].v[p], dxu);
                            s1 = p ? __ffma2_rn(lam[u].v[p], B.v[p], s1) : __fmul2_rn(lam[u].v[p], B.v[p]);
                            lam[u].v[p] = __fmul2_rn(lam[u].v[p], e[i][u].v[p]);
                            const float2 f = __fmul2_rn(lam[u].v[p], before[i][u].v[p]);
                            s2 = p ? __ffma2_rn(f, A2[u].v[p], s2) : __fmul2_rn(f, A2[u].v[p]);
                            dA[u].v[p] = __ffma2_rn(f, dtu, dA[u].v[p]);
                        }
                        into[u][i] = s1.x + s1.y, back[u][i] = s2.x + s2.y, out[u][i] = s3.x + s3.y;
                        now[u] = before[i][u];
                    }
                    float v[2 * SPL];
#pragma unroll
                    for (int p = 0; p < P; ++p) {
                        v[2 * p < SPL ? 2 * p : 0] = gb[p].x;
                        v[SPL + 2 * p < 2 * SPL ? SPL + 2 * p : SPL] = gc[p].x;
                        if (SPL > 1) v[2 * p + 1 < SPL ? 2 * p + 1 : 0] = gb[p].y, v[SPL + 2 * p + 1 < 2 * SPL ? SPL + 2 * p + 1 : SPL] = gc[p].y;
                    }
                    mine[(4 * j + i) * 32] = channel_sums<SPL>(v);
                }
                const float2 slope = kept(kSlope, j);
                float dxv[2], ddv[2], dzv[2];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const float lb = quad_sums(into[u][0], into[u][1], into[u][2], into[u][3]);
                    const float ah = 0.69314718055994531f * quad_sums(back[u][0], back[u][1], back[u][2], back[u][3]);  // (A2 is A log2 e)
                    const float ys = quad_sums(out[u][0], out[u][1], out[u][2], out[u][3]);
                    ddv[u] = 4 * j + q < left ? fmaf(xv[u], lb, ah) * (u ? slope.y : slope.x) : 0.0f;
                    dskip[u] = fmaf(gy[u], xv[u], dskip[u]);
                    dbias[u] += ddv[u];
                    dxv[u] = fmaf(dt[u], lb, skip[u] * gy[u]);
                    dzv[u] = dyv[u] * fmaf(skip[u], xv[u], ys) * gs[u];
                }
                if (on && 4 * j + q < left) {
                    const long long at = out0 + (long long)(t0 + 4 * j + q) * a.D;
                    store_two((T*)a.dx + at, dxv[0], dxv[1], pair, both);
                    store_two((T*)a.ddelta + at, ddv[0], ddv[1], pair, both);
                    if (z) store_two((T*)a.dz + at, dzv[0], dzv[1], pair, both);
                }
            }
            if (c > 0) store_bc(bcs + ((c - 1) & 1) * L::bc);
            __syncthreads();
#pragma unroll
            for (int i = 0; i < kChunk / kGradWarps; ++i) {  // a warp joins the sums of every fourth token
                const int t = i * kGradWarps + w;
                if (t >= left) break;
                float s = 0.0f;
#pragma unroll
                for (int r = 0; r < kGradWarps; ++r) s += red[(c & 1) * L::red + (r * kChunk + t) * 32 + lane];
                k.bc[((long long)tile * a.total + g.first + t0 + t) * 32 + lane] = s;
            }
        }
        if (g.s == 0 && a.dinitial) {
            float* to = a.dinitial + (long long)g.b * DN + (long long)d * a.N + n0;
            if (on) lam[0].store_some(to, n0, a.N);
            if (both) lam[1].store_some(to + a.N, n0, a.N);
        }
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        dskip[u] += __shfl_xor_sync(0xffffffffu, dskip[u], 1), dskip[u] += __shfl_xor_sync(0xffffffffu, dskip[u], 2);
        dbias[u] += __shfl_xor_sync(0xffffffffu, dbias[u], 1), dbias[u] += __shfl_xor_sync(0xffffffffu, dbias[u], 2);
        if (!(u ? both : on)) continue;
        dA[u].store_some(params + (long long)(d + u) * a.N + n0, n0, a.N);
        if (q == 0) params[DN + d + u] = dskip[u], params[DN + a.D + d + u] = dbias[u];
    }
}

// dB and dC: the sums over the tiles of channels; a warp takes a row.  Rows of no sequence are zero.
template <typename T, int NP> __global__ void __launch_bounds__(256) token_scan_bc_kernel(ScanKernel k) {
    constexpr int SPL = NP / 4;
    pdl_wait();
    pdl_launch_dependents();
    const TokenScanArgs& a = k.a;
    if (a.offsets) check_offsets(a, blockIdx.x, gridDim.x);
    const int lane = threadIdx.x & 31;
    const long long row = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (row >= a.total) return;
    float s = 0.0f;
    if (!a.offsets || (row >= a.offsets[0] && row < a.offsets[a.B])) {
        const float* p = k.bc + row * 32 + lane;
#pragma unroll 4
        for (int i = 0; i < k.tiles; ++i) s += p[(long long)i * a.total * 32];
    }
    for (int j = lane; j < 32; j += 32) {
        const bool is_c = j >= 16;
        const int n = j & 15;
        const float v = __shfl_sync(0xffffffffu, s, bc_lane<SPL>(is_c, n < NP ? n : 0));
        if (n < a.N) ((T*)(is_c ? a.dC : a.dB))[row * a.N + n] = io<T>::to(v);
    }
}

// Tokens of a segment of the gradients: such that there are about three CTAs for each that an SM holds, at least two chunks and at
// most 32 segments to a sequence.
int grad_segment(int B, int T, long long total, int D) {
    const long long tiles = (D + kScanCh - 1) / kScanCh, want = 6LL * device_sm_count();
    const int whole = (T + kScanChunk - 1) / kScanChunk * kScanChunk;
    if (T <= 2 * kScanChunk) return whole < kScanChunk ? kScanChunk : whole;
    const long long segs = (want + tiles - 1) / tiles;
    long long seg = (total + segs - 1) / segs;
    if (seg * 32 < T) seg = (T + 31) / 32;
    seg = (seg + kScanChunk - 1) / kScanChunk * kScanChunk;
    if (seg < 2 * kScanChunk) seg = 2 * kScanChunk;
    return (int)(seg < whole ? seg : whole);
}

struct GradLayout {
    size_t local, decay, bc, params, bytes;
};
GradLayout grad_layout(long long slots, int tiles, long long total, int D, int N) {
    GradLayout l;
    l.local = 256;
    l.decay = l.local + align_up((size_t)slots * D * padded_states(N) * 4, 256);
    l.bc = l.decay + align_up((size_t)slots * D * 4, 256);
    l.params = l.bc + align_up((size_t)tiles * total * 32 * 4, 256);
    l.bytes = l.params + align_up((size_t)slots * D * (N + 2) * 4, 256);
    return l;
}

template <typename T, int NP> vmb_status run_grad(const ScanKernel& k0, cudaStream_t stream) {
    ScanKernel k = k0;
    const TokenScanArgs& a = k.a;
    const void *adjoint = (const void*)token_scan_adjoint_kernel<T, NP>, *grad = (const void*)token_scan_grad_kernel<T, NP>;
    constexpr int abytes = AdjointSmem<T, NP>::bytes;
    constexpr int gbytes = GradSmem<NP>::bytes;
    if (cudaFuncSetAttribute(adjoint, cudaFuncAttributeMaxDynamicSharedMemorySize, abytes) != cudaSuccess ||
        cudaFuncSetAttribute(grad, cudaFuncAttributeMaxDynamicSharedMemorySize, gbytes) != cudaSuccess)
        return VMB_ERR_CUDA;
    void* args[] = {&k};
    // (grids below a wave are not launched early: they would fill the SMs that are free first)
    const unsigned first = (unsigned)((long long)k.slots * k.tiles), grid = first + (a.offsets ? (unsigned)(kClearBlocks * k.tiles) : 0u);
    if (k.seg < a.T && launch_kernel(adjoint, dim3(first), dim3(kScanThreads), abytes, args, stream, first >= resident_ctas(adjoint, kScanThreads, abytes)) != cudaSuccess)
        return VMB_ERR_CUDA;
    if (launch_kernel(grad, dim3(grid), dim3(kGradThreads), gbytes, args, stream, grid >= resident_ctas(grad, kGradThreads, gbytes)) != cudaSuccess) return VMB_ERR_CUDA;
    if (a.total > 0 && launch_kernel((const void*)token_scan_bc_kernel<T, NP>, dim3((unsigned)((a.total + 7) / 8)), dim3(256), 0, args, stream) != cudaSuccess)
        return VMB_ERR_CUDA;
    return launch_column_sums(k.params, k.slots, (long long)a.D * (a.N + 2), a.D * a.N, 1, a.dA, a.dskip, a.D, a.dbias, stream);
}

}  // namespace

size_t token_scan_workspace_bytes(int B, int T, long long total, bool packed, int D, int N, bool grads, vmb_dtype) {
    if (!grads) return token_scan_forward_bytes(B, T, total, packed, D, N);
    const long long slots = scan_slots(B, T, total, packed, grad_segment(B, T, total, D));
    return grad_layout(slots, (D + kScanCh - 1) / kScanCh, total, D, N).bytes;
}

vmb_status launch_token_scan_bwd(const TokenScanArgs& a, cudaStream_t stream) {
    ScanKernel k{a};
    token_scan_plan(k, grad_segment(a.B, a.T, a.total, a.D));
    const GradLayout l = grad_layout(k.slots, k.tiles, a.total, a.D, a.N);
    if (a.ws_bytes < l.bytes) return VMB_ERR_WORKSPACE;
    char* ws = (char*)a.ws;
    k.local = (float*)(ws + l.local), k.decay = (float*)(ws + l.decay), k.bc = (float*)(ws + l.bc), k.params = (float*)(ws + l.params);
    if (k.slots == 0) return VMB_OK;
    const int np = padded_states(a.N);
    if (a.dtype == VMB_BF16)
        return np == 16 ? run_grad<__nv_bfloat16, 16>(k, stream) : np == 8 ? run_grad<__nv_bfloat16, 8>(k, stream) : run_grad<__nv_bfloat16, 4>(k, stream);
    return np == 16 ? run_grad<float, 16>(k, stream) : np == 8 ? run_grad<float, 8>(k, stream) : run_grad<float, 4>(k, stream);
}

}  // namespace vmb
