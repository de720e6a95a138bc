// token_scan_grad.cu - gradients of the selective scan over tokens.
//
// With g_t = dy_t silu(z_t) (dy_t without a gate), a_t = exp(dt_t A) and the adjoint of the state
//   lam_t = C_t g_t + a_(t+1) lam_(t+1):
//   dx = dt (lam . B) + D g,   ddt = x (lam . B) + sum_n A a h_(t-1) lam,   ddelta = ddt softplus'(delta + bias),
//   dB = sum_channels lam dt x,   dC = sum_channels g h_t,   dz = dy (C . h + D x) silu'(z),
//   dA = sum_tokens dt a h_(t-1) lam,   dD = sum g x,   dbias = sum ddelta.
//
// The states are formed again from those that the forward kept before every 64 tokens.  A sequence is cut into segments: a first
// launch leaves what each segment's tokens give to the adjoint before it (a sum without a recurrence: the product of the
// decays up to a token is the exponential of A times the sum of the step sizes), and a segment of the second launch starts from
// the joined sums of those behind it.  Three exponentials for each state, and the sums over the channels (a warp's eight by
// shuffles, a CTA's eight warps through shared memory, the tiles by a third launch, in a fixed order) are what bounds it.
#include "token_scan.cuh"

namespace vmb {

namespace {

constexpr int kTok = kScanChunk, kBlk = 8, kBlocks = kTok / kBlk;

// ------------------------------------------------------------ the adjoint of each segment alone

template <typename T, int NP> struct AdjointSmem {
    static constexpr int array = 32 * scan_pitch<T>(), bytes = 3 * array + 32 * 2 * NP * 4;
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
    RowsBC<T, NP, TOK> bc;
    for (int t0 = 0; t0 < g.len; t0 += TOK) {
        const int left = g.len - t0;
        if (t0) __syncthreads();
        stage_rows<T>(smem, dy + (long long)t0 * a.D, a.D, TOK, left, cols, k.vec);
        stage_rows<T>(smem + L::array, raw + t0 * a.d_t, a.d_t, TOK, left, cols, k.vec);
        if (z) stage_rows<T>(smem + 2 * L::array, z + t0 * a.z_t, a.z_t, TOK, left, cols, k.vec);
        bc.load(nullptr, 0, 0, Cm + t0 * a.C_t, a.C_t, a.N, left);
        bc.store(rows);
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
                C.load(rows + (t + u) * 2 * NP + NP + n0);
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

template <typename T, int NP> struct GradSmem {
    static constexpr int array = kTok * scan_pitch<T>(), bc = 4 * array, starts = bc + kTok * 2 * NP * 4,
                         red = starts + kBlocks * kScanThreads * NP, bytes = red + 2 * 8 * kBlk * 32 * 4;
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

template <typename T, int NP> __global__ void __launch_bounds__(kScanThreads, sizeof(T) == 2 ? 2 : 1) token_scan_grad_kernel(ScanKernel k) {
    constexpr int SPL = NP / 4, P = Pairs<SPL>::P;
    using L = GradSmem<T, NP>;
    extern __shared__ __align__(16) char smem[];
    pdl_wait();
    pdl_launch_dependents();
    const TokenScanArgs& a = k.a;
    const int tile = blockIdx.x % k.tiles, tid = threadIdx.x, lane = tid & 31, w = tid >> 5, q = tid & 3, ch = tid >> 2;
    const int c0 = tile * kScanCh, d = c0 + ch, n0 = q * SPL;
    const int cols = min(kScanCh, a.D - c0);
    const long long slot = blockIdx.x / k.tiles;
    if (slot >= k.slots) {  // rows before the first and behind the last sequence (B's and C's are cleared by the sums over the tiles)
        const long long lo = min(max((long long)a.offsets[0], 0LL), a.total), hi = min(max((long long)a.offsets[a.B], lo), a.total);
        for (long long r = slot - k.slots; r < a.total - (hi - lo); r += kClearBlocks)
            for (int c = tid; c < cols; c += kScanThreads) {
                const long long at = (r < lo ? r : r + hi - lo) * a.D + c0 + c;
                ((T*)a.dx)[at] = ((T*)a.ddelta)[at] = io<T>::to(0.0f);
                if (a.z) ((T*)a.dz)[at] = io<T>::to(0.0f);
            }
        return;
    }
    const ScanSegment g = scan_segment(k, slot);
    const bool on = d < a.D;
    const long long DN = (long long)a.D * a.N;
    float* params = k.params + slot * (DN + 2 * a.D);
    Pairs<SPL> A, A2, lam, dA;
    A.zero(), A2.zero(), lam.zero(), dA.zero();
    float dskip = 0.0f, dbias = 0.0f;
    if (g.live) {
        const float *rows = (const float*)(smem + L::bc);
        float* starts = (float*)(smem + L::starts);
        float* red = (float*)(smem + L::red);
        if (on) {
            A.load_some(a.A + (long long)d * a.N + n0, n0, a.N);
#pragma unroll
            for (int p = 0; p < P; ++p) A2.v[p] = __fmul2_rn(A.v[p], twice(kLog2e));
            if (a.dfinal) lam.load_some(a.dfinal + (long long)g.b * DN + (long long)d * a.N + n0, n0, a.N);
            for (int s = g.segs - 1; s > g.s; --s) {
                const long long at = (g.place + s) * a.D + d;
                Pairs<SPL> l, e;
                l.load(k.local + at * NP + n0);
                decays(e, A2, k.decay[at]);
#pragma unroll
                for (int p = 0; p < P; ++p) lam.v[p] = __ffma2_rn(e.v[p], lam.v[p], l.v[p]);
            }
        }
        const float bias = on && a.bias ? a.bias[d] : 0.0f, skip = on && a.skip ? a.skip[d] : 0.0f;
        const T *x = scan_row<T>(a.x, a, g, a.x_b, a.x_t) + c0, *raw = scan_row<T>(a.delta, a, g, a.d_b, a.d_t) + c0;
        const T *z = a.z ? scan_row<T>(a.z, a, g, a.z_b, a.z_t) + c0 : nullptr, *dy = (const T*)a.dy + g.first * a.D + c0;
        const T *Bm = scan_row<T>(a.Bm, a, g, a.B_b, a.B_t), *Cm = scan_row<T>(a.Cm, a, g, a.C_b, a.C_t);
        char *sx = smem, *sr = smem + L::array, *sg = smem + 2 * L::array, *sz = smem + 3 * L::array;
        int turn = 0;
        for (int c = (g.len + kTok - 1) / kTok - 1; c >= 0; --c) {
            const int t0 = c * kTok, left = g.len - t0;
            {
                RowsBC<T, NP, kTok> bc;
                stage_rows<T>(sx, x + t0 * a.x_t, a.x_t, kTok, left, cols, k.vec);
                stage_rows<T>(sr, raw + t0 * a.d_t, a.d_t, kTok, left, cols, k.vec);
                stage_rows<T>(sg, dy + (long long)t0 * a.D, a.D, kTok, left, cols, k.vec);
                if (z) stage_rows<T>(sz, z + t0 * a.z_t, a.z_t, kTok, left, cols, k.vec);
                bc.load(Bm + t0 * a.B_t, a.B_t, a.N, Cm + t0 * a.C_t, a.C_t, a.N, left);
                bc.store((float*)rows);
                cp_async_commit();
            }
            Pairs<SPL> h;
            h.zero();
            if (on) h.load_some(a.saved + ((g.chunk + ((long long)g.s * k.seg + t0) / kScanChunk) * a.D + d) * a.N + n0, n0, a.N);
            cp_async_wait<0>();
            __syncthreads();
            // the states before each block of eight tokens
            for (int b = 0; b < kBlocks; ++b) {
                h.store(starts + (b * kScanThreads + tid) * SPL);
                if (b == kBlocks - 1) break;
#pragma unroll
                for (int o = 0; o < kBlk; o += 4) {
                    const int t = b * kBlk + o;
                    float dt = staged<T>(sr, t + q, ch) + bias;
                    if (a.softplus) dt = softplus(dt);
                    if (t + q >= left) dt = 0.0f;
                    const float dtx = dt * staged<T>(sx, t + q, ch);
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        Pairs<SPL> B, e;
                        const float dxu = from_lane(dtx, u);
                        B.load(rows + (t + u) * 2 * NP + n0);
                        decays(e, A2, from_lane(dt, u));
#pragma unroll
                        for (int p = 0; p < P; ++p) h.v[p] = __ffma2_rn(e.v[p], h.v[p], __fmul2_rn(twice(dxu), B.v[p]));
                    }
                }
            }
            for (int b = kBlocks - 1; b >= 0; --b, turn ^= 1) {
                if (b * kBlk >= left) continue;  // (the same for the whole CTA)
                // this lane's two tokens of the block
                float xv[2], dt[2], dtx[2], gy[2], gs[2], dyv[2], slope[2];
#pragma unroll
                for (int o = 0; o < 2; ++o) {
                    const int t = b * kBlk + 4 * o + q;
                    xv[o] = staged<T>(sx, t, ch);
                    dyv[o] = gy[o] = staged<T>(sg, t, ch);
                    gs[o] = 0.0f;
                    if (z) {
                        const float zv = staged<T>(sz, t, ch), s = logistic(zv);
                        gs[o] = s * fmaf(zv, 1.0f - s, 1.0f);
                        gy[o] *= zv * s;
                    }
                    float v = staged<T>(sr, t, ch) + bias;
                    slope[o] = 1.0f;
                    if (a.softplus) {
                        const float e = softplus_e(v);
                        slope[o] = softplus_grad_from_e(v, e);
                        v = softplus_from_e(v, e);
                    }
                    dt[o] = t < left ? v : 0.0f;
                    dtx[o] = dt[o] * xv[o];
                }
                Pairs<SPL> e[kBlk], before[kBlk];
                h.load(starts + (b * kScanThreads + tid) * SPL);
#pragma unroll
                for (int i = 0; i < kBlk; ++i) {
                    Pairs<SPL> B;
                    const float dxu = from_lane(dtx[i / 4], i % 4);
                    B.load(rows + (b * kBlk + i) * 2 * NP + n0);
                    decays(e[i], A2, from_lane(dt[i / 4], i % 4));
                    before[i] = h;
#pragma unroll
                    for (int p = 0; p < P; ++p) h.v[p] = __ffma2_rn(e[i].v[p], h.v[p], __fmul2_rn(twice(dxu), B.v[p]));
                }
                float into[kBlk], back[kBlk], out[kBlk];
                float* r = red + turn * (8 * kBlk * 32) + w * (kBlk * 32) + lane;
#pragma unroll
                for (int i = kBlk - 1; i >= 0; --i) {
                    const float gu = from_lane(gy[i / 4], i % 4), dtu = from_lane(dt[i / 4], i % 4), dxu = from_lane(dtx[i / 4], i % 4);
                    Pairs<SPL> B, C;
                    B.load(rows + (b * kBlk + i) * 2 * NP + n0);
                    C.load(rows + (b * kBlk + i) * 2 * NP + NP + n0);
                    float2 s1 = make_float2(0.0f, 0.0f), s2 = s1, s3 = s1;
                    float v[2 * SPL];
#pragma unroll
                    for (int p = 0; p < P; ++p) {
                        const float2 now = i == kBlk - 1 ? h.v[p] : before[i + 1 < kBlk ? i + 1 : i].v[p];
                        s3 = __ffma2_rn(C.v[p], now, s3);
                        lam.v[p] = __ffma2_rn(C.v[p], twice(gu), lam.v[p]);
                        const float2 gc = __fmul2_rn(twice(gu), now), gb = __fmul2_rn(lam.v[p], twice(dxu));
                        v[2 * p < SPL ? 2 * p : 0] = gb.x;
                        v[SPL + 2 * p < 2 * SPL ? SPL + 2 * p : SPL] = gc.x;
                        if (SPL > 1) v[2 * p + 1 < SPL ? 2 * p + 1 : 0] = gb.y, v[SPL + 2 * p + 1 < 2 * SPL ? SPL + 2 * p + 1 : SPL] = gc.y;
                        s1 = __ffma2_rn(lam.v[p], B.v[p], s1);
                        lam.v[p] = __fmul2_rn(lam.v[p], e[i].v[p]);
                        const float2 f = __fmul2_rn(lam.v[p], before[i].v[p]);
                        s2 = __ffma2_rn(f, A.v[p], s2);
                        dA.v[p] = __ffma2_rn(f, twice(dtu), dA.v[p]);
                    }
                    r[i * 32] = channel_sums<SPL>(v);
                    into[i] = s1.x + s1.y, back[i] = s2.x + s2.y, out[i] = s3.x + s3.y;
                }
#pragma unroll
                for (int o = 0; o < 2; ++o) {
                    const int t = b * kBlk + 4 * o + q;
                    const float lb = quad_sums(into[4 * o], into[4 * o + 1], into[4 * o + 2], into[4 * o + 3]);
                    const float ah = quad_sums(back[4 * o], back[4 * o + 1], back[4 * o + 2], back[4 * o + 3]);
                    const float ys = quad_sums(out[4 * o], out[4 * o + 1], out[4 * o + 2], out[4 * o + 3]);
                    const float ddelta = t < left ? fmaf(xv[o], lb, ah) * slope[o] : 0.0f;
                    dskip = fmaf(gy[o], xv[o], dskip);
                    dbias += ddelta;
                    restage<T>(sx, t, ch, fmaf(dt[o], lb, skip * gy[o]));
                    restage<T>(sr, t, ch, ddelta);
                    if (z) restage<T>(sz, t, ch, dyv[o] * fmaf(skip, xv[o], ys) * gs[o]);
                }
                __syncthreads();
                {
                    const int t = b * kBlk + w;  // a warp joins the sums of one token
                    if (t < left) {
                        const float* f = red + turn * (8 * kBlk * 32) + w * 32 + lane;
                        float s = 0.0f;
#pragma unroll
                        for (int i = 0; i < 8; ++i) s += f[i * kBlk * 32];
                        k.bc[((long long)tile * a.total + g.first + t0 + t) * 32 + lane] = s;
                    }
                }
            }
            __syncthreads();
            const long long row = (g.first + t0) * a.D + c0;
            unstage_rows<T>((T*)a.dx + row, sx, a.D, kTok, left, cols, k.vec);
            unstage_rows<T>((T*)a.ddelta + row, sr, a.D, kTok, left, cols, k.vec);
            if (z) unstage_rows<T>((T*)a.dz + row, sz, a.D, kTok, left, cols, k.vec);
            __syncthreads();
        }
        if (on && g.s == 0 && a.dinitial) lam.store_some(a.dinitial + (long long)g.b * DN + (long long)d * a.N + n0, n0, a.N);
    }
    dskip += __shfl_xor_sync(0xffffffffu, dskip, 1), dskip += __shfl_xor_sync(0xffffffffu, dskip, 2);
    dbias += __shfl_xor_sync(0xffffffffu, dbias, 1), dbias += __shfl_xor_sync(0xffffffffu, dbias, 2);
    if (!on) return;
    dA.store_some(params + (long long)d * a.N + n0, n0, a.N);
    if (q == 0) params[DN + d] = dskip, params[DN + a.D + d] = dbias;
}

// dB and dC: the sums over the tiles of channels; a warp takes a row.  Rows of no sequence are zero.
template <typename T, int NP> __global__ void __launch_bounds__(256) token_scan_bc_kernel(ScanKernel k) {
    constexpr int SPL = NP / 4;
    pdl_wait();
    pdl_launch_dependents();
    const TokenScanArgs& a = k.a;
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
    constexpr int abytes = AdjointSmem<T, NP>::bytes, gbytes = GradSmem<T, NP>::bytes;
    if (cudaFuncSetAttribute(adjoint, cudaFuncAttributeMaxDynamicSharedMemorySize, abytes) != cudaSuccess ||
        cudaFuncSetAttribute(grad, cudaFuncAttributeMaxDynamicSharedMemorySize, gbytes) != cudaSuccess)
        return VMB_ERR_CUDA;
    void* args[] = {&k};
    const unsigned grid = (unsigned)((long long)k.slots * k.tiles);
    if (k.seg < a.T && launch_kernel(adjoint, dim3(grid), dim3(kScanThreads), abytes, args, stream, grid >= resident_ctas(adjoint, kScanThreads, abytes)) != cudaSuccess) return VMB_ERR_CUDA;
    if (launch_kernel(grad, dim3(grid + (a.offsets ? (unsigned)(kClearBlocks * k.tiles) : 0u)), dim3(kScanThreads), gbytes, args, stream,
                      grid >= resident_ctas(grad, kScanThreads, gbytes)) != cudaSuccess)
        return VMB_ERR_CUDA;
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
