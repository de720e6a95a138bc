// token_scan.cu - the selective scan over tokens, channels last: forward and the step of serving.
//
//   dt = softplus(delta + bias),  h_t = exp(dt A) h_(t-1) + dt x B_t,  y = C_t . h_t + D x,  y silu(z) with a gate.
//
// N exponentials, N / 2 packed products for each of four uses, and two more exponentials for the step size and the gate per
// channel and token bound it: the issue slots and the FMA and MUFU pipes (0.62 of the slots, 0.40 and 0.38 of the pipes), not the bytes.  Sequences too few to fill the SMs are cut into segments:
// a first launch takes each segment from a zero state and leaves its last state and the sum of its step sizes (the product of
// its decays is the exponential of A times that sum), and each segment of the second launch joins those before it.
#include <initializer_list>

#include "token_scan.cuh"

namespace vmb {

namespace {

// Two lanes hold the states of a channel; a CTA takes the 64 channels of a tile.  A lane of the pair reads and prepares one token of every
// two (step size, its product with x, skip, gate), in blocks of 8 tokens whose values were asked for a block before, and hands
// them to the other by shuffles.  B and C of 32 tokens are in shared memory in fp32.
// 38 sequences of 2048 tokens of 1024 channels and 16 states, bf16, with a gate: 438 us, 68 instructions a token, warp and lane pair; one lane for
// a channel takes the same with all SMs full and longer with fewer sequences, four took 939 us.
constexpr int kLanes = 2, kFwdThreads = kLanes * kScanCh, kTok = 32, kBlk = 8, kPer = kTok / kBlk, kMine = kBlk / kLanes;

template <typename T, int NP, bool kLocal> __global__ void __launch_bounds__(kFwdThreads, 4) token_scan_kernel(ScanKernel k) {
    constexpr int SPL = NP / kLanes, P = Pairs<SPL>::P, kEach = kTok * 2 * NP / kFwdThreads;
    __shared__ __align__(16) float bcs[2][kTok * 2 * NP];
    pdl_wait();
    pdl_launch_dependents();
    const TokenScanArgs& a = k.a;
    const int tile = blockIdx.x % k.tiles, tid = threadIdx.x, p = tid & 1, c0 = tile * kScanCh, d = c0 + tid / kLanes, n0 = p * SPL;
    const long long slot = blockIdx.x / k.tiles;
    if (slot >= k.slots) {  // rows before the first and behind the last sequence
        check_offsets(a, (slot - k.slots) * k.tiles + tile, (long long)kClearBlocks * k.tiles);
        const long long lo = min(max((long long)a.offsets[0], 0LL), a.total), hi = min(max((long long)a.offsets[a.B], lo), a.total);
        const int cols = min(kScanCh, a.D - c0);
        for (long long r = slot - k.slots; r < a.total - (hi - lo); r += kClearBlocks)
            for (int c = tid; c < cols; c += kFwdThreads) ((T*)a.y)[(r < lo ? r : r + hi - lo) * a.D + c0 + c] = io<T>::to(0.0f);
        return;
    }
    const ScanSegment g = scan_segment(k, slot);
    if (!g.live || (kLocal && g.s == g.segs - 1)) return;  // (nothing follows the last segment)
    const bool on = d < a.D, gate = !kLocal && a.z;
    const int dd = on ? d : a.D - 1;  // (lanes behind the last channel keep their warp's shuffles whole)
    Pairs<SPL> A2, h;
    A2.load_some(a.A + (long long)dd * a.N + n0, n0, a.N);
#pragma unroll
    for (int i = 0; i < P; ++i) A2.v[i] = __fmul2_rn(A2.v[i], twice(kLog2e));
    h.zero();
    const float bias = a.bias ? a.bias[dd] : 0.0f, skip = !kLocal && a.skip ? a.skip[dd] : 0.0f;
    // this lane's next token of each array, and its value of B or C in this thread's next row of the stage
    const int xs = (int)a.x_t, ds = (int)a.d_t, zs = (int)a.z_t;
    const T *x = scan_row<T>(a.x, a, g, a.x_b, a.x_t) + p * a.x_t + dd, *raw = scan_row<T>(a.delta, a, g, a.d_b, a.d_t) + p * a.d_t + dd;
    const T* z = gate ? scan_row<T>(a.z, a, g, a.z_b, a.z_t) + p * a.z_t + dd : nullptr;
    T* y = (T*)a.y + (g.first + p) * a.D + d;
    constexpr int kRows = kFwdThreads / (2 * NP);
    const int bn = tid % (2 * NP), brow = tid / (2 * NP), bs = (int)(bn < NP ? a.B_t : a.C_t);
    const bool bin = bn < NP ? bn < a.N : !kLocal && bn - NP < a.N;
    const T* bc = bn < NP ? scan_row<T>(a.Bm, a, g, a.B_b, a.B_t) + bn : scan_row<T>(a.Cm, a, g, a.C_b, a.C_t) + (bn - NP);
    bc += (long long)brow * bs;
    const int blocks = (g.len + kBlk - 1) / kBlk;

    T rx[kMine], rd[kMine], rz[kMine], rbc[kEach];
    auto load = [&](int left) {  // `left` tokens, the block's among them (rows behind the last: the last again)
        if (left >= kBlk) {
#pragma unroll
            for (int j = 0; j < kMine; ++j) {
                rx[j] = x[kLanes * j * xs], rd[j] = raw[kLanes * j * ds];
                if (gate) rz[j] = z[kLanes * j * zs];
            }
        } else {
#pragma unroll
            for (int j = 0; j < kMine; ++j) {
                const int t = min(kLanes * j, left - 1 - p);
                rx[j] = x[t * xs], rd[j] = raw[t * ds];
                if (gate) rz[j] = z[t * zs];
            }
        }
        x += (long long)kBlk * xs, raw += (long long)kBlk * ds;
        if (gate) z += (long long)kBlk * zs;
    };
    auto load_bc = [&](int left) {
#pragma unroll
        for (int j = 0; j < kEach; ++j) rbc[j] = bin && brow + j * kRows < left ? bc[j * kRows * bs] : io<T>::to(0.0f);
        bc += (long long)kTok * bs;
    };
    auto store_bc = [&](float* s) {
#pragma unroll
        for (int j = 0; j < kEach; ++j) s[tid + j * kFwdThreads] = io<T>::cvt(rbc[j]);
    };
    if (blocks > 0) {
        load_bc(g.len);
        load(g.len);
    }
    if (!kLocal) {
        if (a.initial) h.load_some(a.initial + ((long long)g.b * a.D + dd) * a.N + n0, n0, a.N);
#pragma unroll 4
        for (int s = 0; s < g.s; ++s) {
            const long long at = (g.place + s) * a.D + dd;
            Pairs<SPL> l, e;
            l.load(k.local + at * NP + n0);
            decays(e, A2, k.decay[at]);
#pragma unroll
            for (int i = 0; i < P; ++i) h.v[i] = __ffma2_rn(e.v[i], h.v[i], l.v[i]);
        }
    }
    if (blocks > 0) store_bc(bcs[0]);
    __syncthreads();
    float sum = 0.0f;  // of this lane's step sizes
    const int from0 = tid & 30, from1 = from0 | 1;
    for (int b = 0; b < blocks; ++b) {
        const int t0 = b * kBlk, left = g.len - t0;
        if (b % kPer == 0) load_bc(left - kTok);
        float dt[kMine], dtx[kMine], out[kMine];
        T zv[kMine];
#pragma unroll
        for (int j = 0; j < kMine; ++j) {
            const float xv = io<T>::cvt(rx[j]);
            dt[j] = io<T>::cvt(rd[j]) + bias;
            if (a.softplus) dt[j] = softplus(dt[j]);
            dtx[j] = dt[j] * xv;
            out[j] = skip * xv;
            if (gate) zv[j] = rz[j];
        }
        if (left < kBlk) {
#pragma unroll
            for (int j = 0; j < kMine; ++j)
                if (kLanes * j + p >= left) dt[j] = dtx[j] = 0.0f;
        }
        if (left > kBlk) load(left - kBlk);
        if (!kLocal && a.saved && on && t0 % kScanSaved == 0) {
            float* to = a.saved + ((g.chunk + ((long long)g.s * k.seg + t0) / kScanSaved) * a.D + d) * a.N + n0;
            if (a.N == NP) h.store(to);  // (16-byte aligned)
            else h.store_some(to, n0, a.N);
        }
        const float* rows = bcs[(b / kPer) & 1] + (b % kPer) * kBlk * 2 * NP + n0;
#pragma unroll
        for (int j = 0; j < kMine; ++j) {
            float part[kLanes];
            if (kLocal) sum += dt[j];
            Pairs<SPL> e[kLanes], in[kLanes];
#pragma unroll
            for (int u = 0; u < kLanes; ++u) {
                const float dtu = __shfl_sync(0xffffffffu, dt[j], u ? from1 : from0), dxu = __shfl_sync(0xffffffffu, dtx[j], u ? from1 : from0);
                in[u].load(rows + (kLanes * j + u) * 2 * NP);
                decays(e[u], A2, dtu);
#pragma unroll
                for (int i = 0; i < P; ++i) in[u].v[i] = __fmul2_rn(twice(dxu), in[u].v[i]);
            }
#pragma unroll
            for (int u = 0; u < kLanes; ++u) {
                Pairs<SPL> C;
                if (!kLocal) C.load(rows + (kLanes * j + u) * 2 * NP + NP);
                float2 acc = make_float2(0.0f, 0.0f);
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    h.v[i] = __ffma2_rn(e[u].v[i], h.v[i], in[u].v[i]);
                    if (!kLocal) acc = i == 0 ? __fmul2_rn(C.v[i], h.v[i]) : __ffma2_rn(C.v[i], h.v[i], acc);
                }
                part[u] = acc.x + acc.y;
            }
            if (!kLocal) out[j] += (p ? part[1] : part[0]) + __shfl_xor_sync(0xffffffffu, p ? part[0] : part[1], 1);
        }
        if (!kLocal) {
            if (gate) {
#pragma unroll
                for (int j = 0; j < kMine; ++j) out[j] *= activate<VMB_ACT_SILU>(io<T>::cvt(zv[j]));
            }
            if (on && left >= kBlk) {
#pragma unroll
                for (int j = 0; j < kMine; ++j) y[kLanes * j * a.D] = io<T>::to(out[j]);
            } else if (on) {
#pragma unroll
                for (int j = 0; j < kMine; ++j)
                    if (kLanes * j + p < left) y[kLanes * j * a.D] = io<T>::to(out[j]);
            }
            y += (long long)kBlk * a.D;
        }
        if (b % kPer == kPer - 1) {
            store_bc(bcs[(b / kPer + 1) & 1]);
            __syncthreads();
        }
    }
    if constexpr (kLocal) {
        sum += __shfl_xor_sync(0xffffffffu, sum, 1);
        if (!on) return;
        const long long at = slot * a.D + d;
        h.store(k.local + at * NP + n0);
        if (p == 0) k.decay[at] = sum;
    } else if (on && a.final && g.s == g.segs - 1) {
        h.store_some(a.final + ((long long)g.b * a.D + d) * a.N + n0, n0, a.N);
    }
}

// A few tokens of every row from the state in its slot, updated in place; four lanes a channel, two rows a thread, whose states are under way
// together and which share A.  Bound by the states' bytes: 256 rows of 2048 channels, 67 MB, 18.3 us (one row a thread
// 22.8, four 25.0; with B and C one by one 19.2).
constexpr int kStepRows = 2;
template <typename T, int NP> __global__ void __launch_bounds__(128) token_scan_step_kernel(TokenScanArgs a, int tiles) {
    constexpr int SPL = NP / 4, P = Pairs<SPL>::P;
    pdl_wait();
    pdl_launch_dependents();
    const int q = threadIdx.x & 3, d = (int)(blockIdx.x % tiles) * 32 + (threadIdx.x >> 2), n0 = q * SPL;
    const long long b0 = (long long)(blockIdx.x / tiles) * kStepRows;
    const bool on = d < a.D;
    const int dd = on ? d : a.D - 1;  // (lanes behind the last channel keep their warp's shuffles whole)
    const bool whole = a.N == NP && (reinterpret_cast<uintptr_t>(a.state) & 15) == 0 && (reinterpret_cast<uintptr_t>(a.A) & 15) == 0;
    // B and C in whole vectors of a lane's states
    const bool vec = a.N == NP && ((a.B_b | a.B_t | a.C_b | a.C_t) & (SPL - 1)) == 0 &&
                     ((reinterpret_cast<uintptr_t>(a.Bm) | reinterpret_cast<uintptr_t>(a.Cm)) & (SPL * sizeof(T) - 1)) == 0;
    const int rows = (int)min((long long)kStepRows, a.B - b0);
    long long slot[kStepRows];
#pragma unroll
    for (int r = 0; r < kStepRows; ++r) {
        slot[r] = -1;
        if (r < rows) slot[r] = a.slots ? a.slots[b0 + r] : b0 + r;
        if (slot[r] >= a.pool) slot[r] = -1;
    }
    Pairs<SPL> A2, h[kStepRows];
    if (whole) A2.load(a.A + (long long)dd * a.N + n0);
    else A2.load_some(a.A + (long long)dd * a.N + n0, n0, a.N);
#pragma unroll
    for (int r = 0; r < kStepRows; ++r) {
        h[r].zero();
        if (slot[r] < 0) continue;
        const float* state = a.state + (slot[r] * a.D + dd) * a.N + n0;
        if (whole) h[r].load(state);
        else h[r].load_some(state, n0, a.N);
    }
#pragma unroll
    for (int p = 0; p < P; ++p) A2.v[p] = __fmul2_rn(A2.v[p], twice(kLog2e));
    const float bias = a.bias ? a.bias[dd] : 0.0f, skip = a.skip ? a.skip[dd] : 0.0f;
    for (int t = 0; t < a.T; ++t) {
        float xv[kStepRows], dt[kStepRows], zv[kStepRows];
        Pairs<SPL> B[kStepRows], C[kStepRows];
#pragma unroll
        for (int r = 0; r < kStepRows; ++r) {
            xv[r] = dt[r] = zv[r] = 0.0f;
            B[r].zero(), C[r].zero();
            if (slot[r] < 0) continue;
            const long long b = b0 + r;
            xv[r] = io<T>::ld((const T*)a.x + b * a.x_b + t * a.x_t + dd);
            dt[r] = io<T>::ld((const T*)a.delta + b * a.d_b + t * a.d_t + dd);
            if (a.z) zv[r] = io<T>::ld((const T*)a.z + b * a.z_b + t * a.z_t + dd);
            const T *Bm = (const T*)a.Bm + b * a.B_b + t * a.B_t + n0, *Cm = (const T*)a.Cm + b * a.C_b + t * a.C_t + n0;
            if (vec) {
                float v[SPL];
                load_vec<T, SPL>(v, Bm);
#pragma unroll
                for (int p = 0; p < P; ++p) B[r].v[p] = make_float2(v[2 * p], SPL > 1 ? v[2 * p + (SPL > 1)] : 0.0f);
                load_vec<T, SPL>(v, Cm);
#pragma unroll
                for (int p = 0; p < P; ++p) C[r].v[p] = make_float2(v[2 * p], SPL > 1 ? v[2 * p + (SPL > 1)] : 0.0f);
                continue;
            }
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const bool one = n0 + 2 * p < a.N, two = SPL > 1 && n0 + 2 * p + 1 < a.N;
                B[r].v[p] = make_float2(one ? io<T>::ld(Bm + 2 * p) : 0.0f, two ? io<T>::ld(Bm + 2 * p + 1) : 0.0f);
                C[r].v[p] = make_float2(one ? io<T>::ld(Cm + 2 * p) : 0.0f, two ? io<T>::ld(Cm + 2 * p + 1) : 0.0f);
            }
        }
#pragma unroll
        for (int r = 0; r < kStepRows; ++r) {
            if (r >= rows) break;  // (the same for the whole block)
            float step = dt[r] + bias;
            if (a.softplus) step = softplus(step);
            Pairs<SPL> e;
            decays(e, A2, step);
            float2 acc = make_float2(0.0f, 0.0f);
#pragma unroll
            for (int p = 0; p < P; ++p) {
                h[r].v[p] = __ffma2_rn(e.v[p], h[r].v[p], __fmul2_rn(twice(step * xv[r]), B[r].v[p]));
                acc = __ffma2_rn(C[r].v[p], h[r].v[p], acc);
            }
            float out = acc.x + acc.y;
            out += __shfl_xor_sync(0xffffffffu, out, 1);
            out += __shfl_xor_sync(0xffffffffu, out, 2);
            out = fmaf(skip, xv[r], out);
            if (a.z) out *= activate<VMB_ACT_SILU>(zv[r]);
            if (on && q == 0) ((T*)a.y)[((b0 + r) * a.T + t) * a.D + d] = io<T>::to(slot[r] < 0 ? 0.0f : out);
        }
    }
    if (!on) return;
#pragma unroll
    for (int r = 0; r < kStepRows; ++r) {
        if (slot[r] < 0) continue;
        float* state = a.state + (slot[r] * a.D + d) * a.N + n0;
        if (whole) h[r].store(state);
        else h[r].store_some(state, n0, a.N);
    }
}

bool vec16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

template <typename T, int NP> vmb_status run_scan(const ScanKernel& k0, unsigned grid, bool cut, cudaStream_t stream) {
    ScanKernel k = k0;
    const void *local = (const void*)token_scan_kernel<T, NP, true>, *full = (const void*)token_scan_kernel<T, NP, false>;
    void* args[] = {&k};
    const unsigned first = (unsigned)((long long)k.slots * k.tiles);
    // (grids below a wave are not launched early: they would fill the SMs that are free first)
    if (cut && launch_kernel(local, dim3(first), dim3(kFwdThreads), 0, args, stream, first >= resident_ctas(local, kFwdThreads, 0)) != cudaSuccess)
        return VMB_ERR_CUDA;
    return launch_kernel(full, dim3(grid), dim3(kFwdThreads), 0, args, stream, grid >= resident_ctas(full, kFwdThreads, 0)) == cudaSuccess ? VMB_OK : VMB_ERR_CUDA;
}
template <typename T> vmb_status run_scan(const ScanKernel& k, unsigned grid, bool cut, cudaStream_t stream) {
    const int np = padded_states(k.a.N);
    return np == 4 ? run_scan<T, 4>(k, grid, cut, stream) : np == 8 ? run_scan<T, 8>(k, grid, cut, stream) : run_scan<T, 16>(k, grid, cut, stream);
}

// Tokens of a forward segment, a multiple of 64.  Dense: by estimated clocks.  With one to four CTAs on an SM a token takes 248, 262, 330 or
// 395 of them (measured with 16 states and a gate; the third in between), and no more than four fit; cut sequences take 1.7 times that, for the first launch, and
// 12000 for its start and the joins.  19 sequences of 1024 channels, two CTAs on each SM, stay whole (291 us, cut in three 359); of 512
// channels, one on each, are cut (192 us, whole 275); a single one of 3136 tokens and 384 channels is cut in 49 (29 us, in 25 33, whole 295).
// Packed: their lengths are not known here, the long ones are cut for balance, eight segments for each SM (24 of 1 to 4096 tokens and 1536
// channels: 368 us, with four for each SM 428, whole 631).
int forward_segment(int B, int T, long long total, bool packed, int D) {
    const long long tiles = (D + kScanCh - 1) / kScanCh, sms = device_sm_count();
    const auto chunks = [](long long t) { return t < 1 ? (long long)kScanChunk : (t + kScanChunk - 1) / kScanChunk * kScanChunk; };
    if (packed) {
        const long long segs = (8 * sms + tiles - 1) / tiles, seg = chunks((total + segs - 1) / segs), least = chunks((total + 63) / 64);
        return (int)(seg > least ? seg : least);
    }
    const double per_token[4] = {248.0, 262.0, 330.0, 395.0};
    long long best = chunks(T);
    double least = -1.0;
    for (int want = 1; want <= 64 && (want == 1 || best > kScanChunk); ++want) {
        const long long seg = chunks((T + want - 1) / want), segs = (T + seg - 1) / seg, ctas = (long long)B * tiles * (segs > 1 ? segs : 1);
        const long long full = ctas / (4 * sms), rest = ctas % (4 * sms);
        const double token = 395.0 * full + (rest ? per_token[(rest + sms - 1) / sms - 1] : 0.0);
        const double clocks = seg * token * (segs > 1 ? 1.7 : 1.0) + (segs > 1 ? 12000.0 : 0.0);
        if (least < 0.0 || clocks < least) least = clocks, best = seg;
    }
    return (int)best;
}

}  // namespace

void token_scan_plan(ScanKernel& k, int seg) {
    const TokenScanArgs& a = k.a;
    k.seg = seg;
    k.segs_per = (a.T + seg - 1) / seg;
    if (k.segs_per < 1) k.segs_per = 1;
    k.slots = (int)(a.offsets ? scan_slots(a.B, a.T, a.total, true, seg) : (long long)a.B * k.segs_per);
    k.tiles = (a.D + kScanCh - 1) / kScanCh;
    const int V = a.dtype == VMB_BF16 ? 8 : 4;
    k.vec = a.D % V == 0 && a.x_t % V == 0 && a.d_t % V == 0 && (!a.z || a.z_t % V == 0) && vec16(a.x) && vec16(a.delta) && vec16(a.z) &&
            vec16(a.y) && vec16(a.dy) && vec16(a.dx) && vec16(a.ddelta) && vec16(a.dz);
    if (!a.offsets && a.B > 1) k.vec = k.vec && a.x_b % V == 0 && a.d_b % V == 0 && (!a.z || a.z_b % V == 0);
    const size_t two = a.dtype == VMB_BF16 ? 3 : 7;
    k.pair = ((a.D | a.x_t | a.d_t | a.z_t) & 1) == 0;
    for (const void* p : {a.x, a.delta, a.z, a.dy, (const void*)a.dx, (const void*)a.ddelta, (const void*)a.dz})
        k.pair = k.pair && (reinterpret_cast<uintptr_t>(p) & two) == 0;
    if (!a.offsets && a.B > 1) k.pair = k.pair && ((a.x_b | a.d_b | a.z_b) & 1) == 0;
}

size_t token_scan_forward_bytes(int B, int T, long long total, bool packed, int D, int N) {
    const int seg = forward_segment(B, T, total, packed, D);
    const long long slots = scan_slots(B, T, total, packed, seg);
    return 256 + align_up((size_t)slots * D * padded_states(N) * 4, 256) + align_up((size_t)slots * D * 4, 256);
}

vmb_status launch_token_scan_fwd(const TokenScanArgs& a, cudaStream_t stream) {
    ScanKernel k{a};
    token_scan_plan(k, forward_segment(a.B, a.T, a.total, a.offsets != nullptr, a.D));
    if (a.ws_bytes < token_scan_forward_bytes(a.B, a.T, a.total, a.offsets != nullptr, a.D, a.N)) return VMB_ERR_WORKSPACE;
    k.local = (float*)((char*)a.ws + 256);
    k.decay = (float*)((char*)k.local + align_up((size_t)k.slots * a.D * padded_states(a.N) * 4, 256));
    const bool cut = k.seg < a.T;
    const unsigned grid = (unsigned)(((long long)k.slots + (a.offsets ? kClearBlocks : 0)) * k.tiles);
    if (grid == 0) return VMB_OK;
    return a.dtype == VMB_BF16 ? run_scan<__nv_bfloat16>(k, grid, cut, stream) : run_scan<float>(k, grid, cut, stream);
}

vmb_status launch_token_scan_step(const TokenScanArgs& a, cudaStream_t stream) {
    TokenScanArgs g = a;
    int tiles = (a.D + 31) / 32;
    void* args[] = {&g, &tiles};
    const int np = padded_states(a.N);
    const void* fn;
    if (a.dtype == VMB_BF16)
        fn = np == 16  ? (const void*)token_scan_step_kernel<__nv_bfloat16, 16>
             : np == 8 ? (const void*)token_scan_step_kernel<__nv_bfloat16, 8>
                       : (const void*)token_scan_step_kernel<__nv_bfloat16, 4>;
    else
        fn = np == 16  ? (const void*)token_scan_step_kernel<float, 16>
             : np == 8 ? (const void*)token_scan_step_kernel<float, 8>
                       : (const void*)token_scan_step_kernel<float, 4>;
    return launch_kernel(fn, dim3((unsigned)(((long long)a.B + kStepRows - 1) / kStepRows * tiles)), dim3(128), 0, args, stream) == cudaSuccess ? VMB_OK : VMB_ERR_CUDA;
}

}  // namespace vmb
