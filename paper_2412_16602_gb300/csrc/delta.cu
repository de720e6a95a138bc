// delta.cu - the gated delta rule: plans, the kernel that joins the segments of a chain, the sum over
// shared heads, the rows that no sequence holds, and the recurrent step.
#include "delta_grad.cuh"
#include "delta_internal.h"
#include "vmb_internal.h"

#include <mutex>

namespace vmb {

namespace {

// ------------------------------------------------------------------ joining segments

// One CTA per chain and 8 rows of the transposed state: S' = S X + N from segment to segment (X the
// segment's map, in reverse its transpose, which the chains store for this), fp32.  The sums N are
// replaced by the state at each segment's start (in reverse: the gradient of the state at its end).
// A serial walk, bound by the latency of a step: every value of a map is used by one thread, which
// reads it from the L2 cache one (Dk > 64) or three steps ahead into registers; a group of Dk / 4
// threads takes every KG-th row of the map for all 8 rows of the state, and the groups' sums meet in
// shared memory.
constexpr int kJoinThreads = 256, kJoinRows = 8;
template <int DK> __global__ void __launch_bounds__(kJoinThreads, 1) delta_join_kernel(DeltaChain c, int reverse) {
    constexpr int L = DK / 4, KG = kJoinThreads / L, E = DK / KG, D = DK == 64 ? 4 : 2, LD = DK + 4;
    __shared__ __align__(16) float S[DK * kJoinRows];         // [column][row]
    __shared__ __align__(16) float part[KG * kJoinRows * LD]; // rows four words apart in the banks
    const DeltaArgs& a = c.a;
    const int tid = threadIdx.x, col = 4 * (tid % L), group = tid / L;
    pdl_launch_dependents();
    pdl_wait();
    const int strips = (a.Dv + kJoinRows - 1) / kJoinRows;
    const long long chain = blockIdx.x / strips;
    // the state's values that this thread carries: four columns of one row
    const int r = tid & 7, oc = 4 * (tid >> 3), row = (int)(blockIdx.x % strips) * kJoinRows + r;
    const bool own = oc < DK, live = own && row < a.Dv;
    const DeltaSeq seq = delta_seq(a.offsets, (int)(chain / a.Hv), a.T, a.total, c.err);
    const int nseg = (chunks_of(seq.len) + c.seg_chunks - 1) / c.seg_chunks;
    const float* init = reverse ? a.dfinal : a.initial;
    float* last = reverse ? a.dinitial : a.final;
    auto sums = [&](int i) { return reinterpret_cast<float4*>(c.sums + ((chain * c.segs + (reverse ? nseg - 1 - i : i)) * a.Dv + row) * DK + oc); };
    float4 m[D][E], n[D];
    auto fetch = [&](int i, float4(&x)[E], float4& y) {
        if (i >= nseg) return;
        const float* p = c.maps + ((chain * c.segs + (reverse ? nseg - 1 - i : i)) * DK + group) * DK + col;
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = *reinterpret_cast<const float4*>(p + e * KG * DK);
        y = live ? *sums(i) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    };
#pragma unroll
    for (int u = 0; u < D - 1; ++u) fetch(u, m[u], n[u]);
    float s[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) s[j] = init && live && oc + j < a.Dk ? init[(chain * a.Dk + oc + j) * a.Dv + row] : 0.0f;
    for (int i0 = 0; i0 < nseg; i0 += D) {
#pragma unroll
        for (int u = 0; u < D; ++u) {
            const int i = i0 + u;
            if (i >= nseg) break;
            if (own) {
#pragma unroll
                for (int j = 0; j < 4; ++j) S[(oc + j) * kJoinRows + r] = s[j];
            }
            if (live) *sums(i) = make_float4(s[0], s[1], s[2], s[3]);
            __syncthreads();
            fetch(i + D - 1, m[(u + D - 1) % D], n[(u + D - 1) % D]);
            float2 acc[kJoinRows][2] = {};
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float4* q = reinterpret_cast<const float4*>(S + (e * KG + group) * kJoinRows);
                const float4 q0 = q[0], q1 = q[1];
                const float v[kJoinRows] = {q0.x, q0.y, q0.z, q0.w, q1.x, q1.y, q1.z, q1.w};
#pragma unroll
                for (int j = 0; j < kJoinRows; ++j) {
                    acc[j][0] = __ffma2_rn(make_float2(v[j], v[j]), make_float2(m[u][e].x, m[u][e].y), acc[j][0]);
                    acc[j][1] = __ffma2_rn(make_float2(v[j], v[j]), make_float2(m[u][e].z, m[u][e].w), acc[j][1]);
                }
            }
#pragma unroll
            for (int j = 0; j < kJoinRows; ++j)
                *reinterpret_cast<float4*>(part + (group * kJoinRows + j) * LD + col) = make_float4(acc[j][0].x, acc[j][0].y, acc[j][1].x, acc[j][1].y);
            __syncthreads();
            if (own) {
                s[0] = n[u].x, s[1] = n[u].y, s[2] = n[u].z, s[3] = n[u].w;
#pragma unroll
                for (int k = 0; k < KG; ++k) {
                    const float4 t = *reinterpret_cast<const float4*>(part + (k * kJoinRows + r) * LD + oc);
                    s[0] += t.x, s[1] += t.y, s[2] += t.z, s[3] += t.w;
                }
            }
        }
    }
    if (last && live) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (oc + j < a.Dk) last[(chain * a.Dk + oc + j) * a.Dv + row] = s[j];
    }
}

// ------------------------------------------------------------------ shared heads

// dq and dk of a key head in fp32: the sum, in order, of those of its value heads.  The CTAs go by chunks (kShareCtas to
// one), so that rows which no sequence holds, and whose parts nothing has written, are left alone.
constexpr int kShareCtas = 16;
__global__ void __launch_bounds__(256) delta_share_kernel(DeltaGrad c) {
    const DeltaArgs& a = c.a;
    pdl_launch_dependents();
    pdl_wait();
    const int chunks = chunks_of(a.T), ch = blockIdx.x % chunks, r = a.Hv / a.Hk, Dk = a.Dk, row = a.Hk * Dk;
    const DeltaSeq seq = delta_seq(a.offsets, blockIdx.x / chunks, a.T, a.total, nullptr);
    constexpr int kRows = kChunk / kShareCtas;
    const int t0 = blockIdx.y * kRows, n = max(0, min(seq.len - ch * kChunk - t0, kRows)) * row;
    const long long token = seq.start + (long long)ch * kChunk + t0;
    const float* part = c.part + token * a.Hv * 2 * Dk;
    float *dq = (float*)a.dq + token * row, *dk = (float*)a.dk + token * row;
    for (int i = threadIdx.x; i < n; i += 256) {
        const float* p = part + (long long)(i / Dk) * r * 2 * Dk + i % Dk;  // i / Dk: (token, key head)
        float q = 0.0f, k = 0.0f;
        for (int j = 0; j < r; ++j) q += p[(long long)j * 2 * Dk], k += p[(long long)j * 2 * Dk + Dk];
        dq[i] = q;
        dk[i] = k;
    }
}

// ------------------------------------------------------------------ rows that no sequence holds

// Zeros in the rows before the first packed sequence, behind the last one (the padding of a token buffer) and between them
// (where one is longer than the stated bound).  The rows at the ends are shared by all CTAs; launched before the
// chains, so that offsets out of order, which make these rows overlap a sequence's, cost no result.
struct DeltaClear {
    const int* offsets;
    int B, T;
    long long total;
    char* p[5];
    long long row[5];  // bytes of a token, a multiple of two
};
__device__ __forceinline__ void clear_bytes(char* p, long long n, long long i0, long long step) {
    const long long odd = (16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15, head = odd < n ? odd : n, words = (n - head) / 16;
    for (long long i = i0; i < head / 2; i += step) reinterpret_cast<unsigned short*>(p)[i] = 0;
    for (long long i = i0; i < words; i += step) reinterpret_cast<uint4*>(p + head)[i] = make_uint4(0, 0, 0, 0);
    p += head + 16 * words;
    for (long long i = i0; i < (n - head - 16 * words) / 2; i += step) reinterpret_cast<unsigned short*>(p)[i] = 0;
}
__global__ void __launch_bounds__(256) delta_clear_kernel(DeltaClear c) {
    pdl_launch_dependents();
    pdl_wait();
    auto clear = [&](long long r0, long long r1, long long i0, long long step) {
        if (r1 <= r0) return;
#pragma unroll
        for (int k = 0; k < 5; ++k)
            if (c.p[k]) clear_bytes(c.p[k] + r0 * c.row[k], (r1 - r0) * c.row[k], i0, step);
    };
    auto seq = [&](int b) { return delta_seq(c.offsets, b, c.T, c.total, nullptr); };
    const long long thread = (long long)blockIdx.x * 256 + threadIdx.x, threads = (long long)gridDim.x * 256;
    const DeltaSeq last = seq(c.B - 1);
    clear(0, seq(0).start, thread, threads);
    clear(last.start + last.len, c.total, thread, threads);
    for (int b = blockIdx.x; b < c.B - 1; b += gridDim.x) {
        const DeltaSeq s = seq(b);
        clear(s.start + s.len, seq(b + 1).start, threadIdx.x, 256);
    }
}

// ------------------------------------------------------------------ the recurrent step

// One warp per 16 value channels of a head: lane (p = lane / 4, c = lane % 4) holds rows 8i + p of the state for channels
// 4c .. 4c + 3, so that the state is read once and written once and the sums over the rows take three shuffles.  One
// pass over the old state gives both S^T k and S^T q:
//   S_t^T q = a S^T q + (q.k) u,  u = b (v - a S^T k).
// Bound by the state's bytes (8 Dk Dv per row of the batch and head): 60.6 us for 256 streams of 12 heads of 128 x 128, 92%
// of the copy rate; one stream of 6 heads of 64 x 64 takes 2.5 us on the device, less than its launch.  (32 channels per
// warp, twice the registers: 73.6 us for the 256 streams; with streaming cache hints 75.9 us.)
template <typename T, int RPL>
__global__ void __launch_bounds__(128) delta_step_kernel(DeltaStep a) {
    __shared__ float2 qk[8 * RPL];
    __shared__ float red[4];
    pdl_launch_dependents();
    pdl_wait();
    const int tid = threadIdx.x, w = tid >> 5, lane = tid & 31, p = lane >> 2, c = (lane & 3) * 4;
    const int groups = (a.Dv + 63) / 64;
    const int grp = blockIdx.x % groups;
    const long long bh = blockIdx.x / groups;
    const int h = (int)(bh % a.Hv), b = (int)(bh / a.Hv), hk = h / (a.Hv / a.Hk);
    const int v0 = grp * 64 + w * 16 + c;
    const long long slot = a.slots ? a.slots[b] : b;
    T* op = (T*)a.o + ((long long)b * a.T * a.Hv + h) * a.Dv;
    if (slot < 0 || slot >= a.pool) {  // no state: a row of padding
        for (int t = 0; t < a.T; ++t)
            if (tid < 64 && grp * 64 + tid < a.Dv) op[(long long)t * a.Hv * a.Dv + grp * 64 + tid] = io<T>::to(0.0f);
        return;
    }
    float* sp = a.state + (slot * a.Hv + h) * a.Dk * a.Dv + v0;
    const bool vec = a.Dv % 4 == 0 && (reinterpret_cast<uintptr_t>(a.state) & 15) == 0;
    float4 S[RPL];
#pragma unroll
    for (int i = 0; i < RPL; ++i) {
        const int d = 8 * i + p;
        S[i] = make_float4(0, 0, 0, 0);
        if (d >= a.Dk) continue;
        const float* s = sp + (long long)d * a.Dv;
        if (vec) {
            if (v0 < a.Dv) S[i] = *reinterpret_cast<const float4*>(s);
        } else {
            if (v0 < a.Dv) S[i].x = s[0];
            if (v0 + 1 < a.Dv) S[i].y = s[1];
            if (v0 + 2 < a.Dv) S[i].z = s[2];
            if (v0 + 3 < a.Dv) S[i].w = s[3];
        }
    }
    for (int t = 0; t < a.T; ++t) {
        const T* qp = (const T*)a.q + b * a.q_b + t * a.q_t + (long long)hk * a.Dk;
        const T* kp = (const T*)a.k + b * a.k_b + t * a.k_t + (long long)hk * a.Dk;
        const T* vp = (const T*)a.v + b * a.v_b + t * a.v_t + (long long)h * a.Dv;
        const long long gi = ((long long)b * a.T + t) * a.Hv + h;
        const float gain = expf(io<T>::cvt(((const T*)a.g)[gi])), beta = io<T>::cvt(((const T*)a.beta)[gi]);
        float v[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) v[x] = v0 + x < a.Dv ? io<T>::cvt(vp[v0 + x]) : 0.0f;
        if (t) __syncthreads();  // the previous token's q and k have been read
        float dot = 0.0f;
        if (tid < 8 * RPL) {
            float2 x = make_float2(0, 0);
            if (tid < a.Dk) x = make_float2(io<T>::cvt(qp[tid]), io<T>::cvt(kp[tid]));
            qk[tid] = x;
            dot = x.x * x.y;
        }
#pragma unroll
        for (int d = 16; d; d >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, d);
        if (lane == 0) red[w] = dot;
        __syncthreads();
        dot = (red[0] + red[1]) + (red[2] + red[3]);
        float4 sk = make_float4(0, 0, 0, 0), sq = sk;
#pragma unroll
        for (int i = 0; i < RPL; ++i) {
            const float2 x = qk[8 * i + p];
            sq.x = fmaf(S[i].x, x.x, sq.x), sq.y = fmaf(S[i].y, x.x, sq.y), sq.z = fmaf(S[i].z, x.x, sq.z), sq.w = fmaf(S[i].w, x.x, sq.w);
            sk.x = fmaf(S[i].x, x.y, sk.x), sk.y = fmaf(S[i].y, x.y, sk.y), sk.z = fmaf(S[i].z, x.y, sk.z), sk.w = fmaf(S[i].w, x.y, sk.w);
        }
#pragma unroll
        for (int d = 4; d <= 16; d <<= 1) {
            sk.x += __shfl_xor_sync(0xffffffffu, sk.x, d), sk.y += __shfl_xor_sync(0xffffffffu, sk.y, d);
            sk.z += __shfl_xor_sync(0xffffffffu, sk.z, d), sk.w += __shfl_xor_sync(0xffffffffu, sk.w, d);
            sq.x += __shfl_xor_sync(0xffffffffu, sq.x, d), sq.y += __shfl_xor_sync(0xffffffffu, sq.y, d);
            sq.z += __shfl_xor_sync(0xffffffffu, sq.z, d), sq.w += __shfl_xor_sync(0xffffffffu, sq.w, d);
        }
        const float4 u = make_float4(beta * (v[0] - gain * sk.x), beta * (v[1] - gain * sk.y), beta * (v[2] - gain * sk.z),
                                     beta * (v[3] - gain * sk.w));
#pragma unroll
        for (int i = 0; i < RPL; ++i) {
            const float k = qk[8 * i + p].y;
            S[i].x = fmaf(gain, S[i].x, k * u.x), S[i].y = fmaf(gain, S[i].y, k * u.y);
            S[i].z = fmaf(gain, S[i].z, k * u.z), S[i].w = fmaf(gain, S[i].w, k * u.w);
        }
        // four of the eight lanes of a channel quad write one channel each
        const float os = p == 0 ? fmaf(gain, sq.x, dot * u.x) : p == 1 ? fmaf(gain, sq.y, dot * u.y)
                       : p == 2 ? fmaf(gain, sq.z, dot * u.z) : fmaf(gain, sq.w, dot * u.w);
        if (p < 4 && v0 + p < a.Dv) op[(long long)t * a.Hv * a.Dv + v0 + p] = io<T>::to(a.scale * os);
    }
#pragma unroll
    for (int i = 0; i < RPL; ++i) {
        const int d = 8 * i + p;
        if (d >= a.Dk) continue;
        float* s = sp + (long long)d * a.Dv;
        if (vec) {
            if (v0 < a.Dv) *reinterpret_cast<float4*>(s) = S[i];
        } else {
            if (v0 < a.Dv) s[0] = S[i].x;
            if (v0 + 1 < a.Dv) s[1] = S[i].y;
            if (v0 + 2 < a.Dv) s[2] = S[i].z;
            if (v0 + 3 < a.Dv) s[3] = S[i].w;
        }
    }
}

vmb_status chain(const DeltaChain& c, bool reverse, cudaStream_t stream) {
    return c.a.dtype == VMB_BF16 ? launch_chain_bf16(c, reverse, stream) : launch_chain_f32(c, reverse, stream);
}

vmb_status join(const DeltaChain& c, bool reverse, cudaStream_t stream) {
    const int strips = (c.a.Dv + kJoinRows - 1) / kJoinRows;
    const void* fn = c.a.Dk <= 64 ? (const void*)delta_join_kernel<64> : (const void*)delta_join_kernel<128>;
    DeltaChain arg = c;
    int rev = reverse;
    void* args[] = {&arg, &rev};
    return launch_kernel(fn, dim3((unsigned)(c.a.B * (long long)c.a.Hv * strips)), dim3(kJoinThreads), 0, args, stream) == cudaSuccess
               ? VMB_OK : VMB_ERR_CUDA;
}

// Of packed sequences: the rows of the outputs that none of them holds.
vmb_status clear(const DeltaArgs& a, bool grads, cudaStream_t stream) {
    if (!a.offsets) return VMB_OK;
    const long long es = a.dtype == VMB_BF16 ? 2 : 4, keys = es * a.Hk * a.Dk, values = es * a.Hv * a.Dv, heads = es * a.Hv;
    DeltaClear c = grads ? DeltaClear{a.offsets, a.B, a.T, a.total, {(char*)a.dq, (char*)a.dk, (char*)a.dv, (char*)a.dg, (char*)a.dbeta},
                                      {keys, keys, values, heads, heads}}
                         : DeltaClear{a.offsets, a.B, a.T, a.total, {(char*)a.o}, {values}};
    void* args[] = {&c};
    return launch_kernel((const void*)delta_clear_kernel, dim3((unsigned)device_sm_count()), dim3(256), 0, args, stream) == cudaSuccess
               ? VMB_OK : VMB_ERR_CUDA;
}

DeltaChain chain_of(const DeltaArgs& a, const DeltaPlan& p) {
    DeltaChain c{};
    c.a = a;
    c.segs = p.segs;
    c.seg_chunks = p.seg_chunks;
    c.wide = p.wide;
    unsigned char* ws = (unsigned char*)a.ws;
    c.maps = (float*)(ws + p.maps_off);
    c.sums = (float*)(ws + p.sums_off);
    c.ds = ws + p.ds_off;
    c.dx = ws + p.dx_off;
    c.err = a.offsets ? &reinterpret_cast<WsHeader*>(a.ws)->err : nullptr;
    return c;
}

}  // namespace

// (the attribute costs about 1 us of host time to set: once per kernel and device)
bool allow_smem(const void* fn, int bytes) {
    struct Entry {
        const void* fn;
        int dev;
    };
    constexpr int kMax = 256;  // above the number of kernel instances; a full table only stops keeping answers
    static std::mutex mu;
    static Entry table[kMax];
    static int used = 0;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return false;
    std::lock_guard<std::mutex> g(mu);
    for (int i = 0; i < used; ++i)
        if (table[i].fn == fn && table[i].dev == dev) return true;
    if (cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) return false;
    if (used < kMax) table[used++] = {fn, dev};
    return true;
}

long long delta_slots(int B, int T, long long total, bool packed) {
    return packed ? total / kChunk + B : (long long)B * chunks_of(T);
}

DeltaPlan plan_delta(const DeltaArgs& a, bool grads, int sms) {
    DeltaPlan p{};
    const long long chains = (long long)a.B * a.Hv;
    p.chunks = chunks_of(a.T);
    p.wide = a.dtype == VMB_BF16 && a.Dv > 64;
    p.slots = delta_slots(a.B, a.T, a.total, a.offsets != nullptr);
    p.segs = 1;
    p.seg_chunks = p.chunks;
    const long long ctas = chains * ((a.Dv + (p.wide ? 127 : 63)) / (p.wide ? 128 : 64));
    // Segments cost a second pass over the chunks, with Dk more rows in it, and the walk that joins them.  Two chunks each or
    // more; taken where they fill the SMs at least four times better, three times for sequences of 64 chunks.  Measured with
    // and without: 36 CTAs (chains and slices of 64 or 128 channels) of 1568 tokens 165 and 212 us in fp32 (64 channels), 70 and
    // 76 in bf16 (64), 173 and 165 (128); 48 CTAs 217 and 212, 85 and 77, 207 and 165, but for 4096 tokens 485 and 533, 178
    // and 199, 404 and 409; 54 CTAs of 4096 tokens, two segments each, 635 and 542, 241 and 202, 538 and 409.
    if (ctas * (p.chunks >= 64 ? 3 : 4) <= sms && p.chunks >= 4) {
        long long segs = sms / ctas;
        if (segs > (p.chunks + 1) / 2) segs = (p.chunks + 1) / 2;
        if (segs > 1) {
            p.seg_chunks = (int)((p.chunks + segs - 1) / segs);
            p.segs = (p.chunks + p.seg_chunks - 1) / p.seg_chunks;
        }
    }
    const size_t es = a.dtype == VMB_BF16 ? 2 : 4;
    size_t at = 256;
    p.maps_off = at;
    const size_t dk = a.Dk <= 64 ? 64 : 128;  // columns of the kernels' states, zeros behind Dk
    if (p.segs > 1) at += align_up((size_t)chains * p.segs * dk * dk * 4, 256);
    p.sums_off = at;
    if (p.segs > 1) at += align_up((size_t)chains * p.segs * a.Dv * dk * 4, 256);
    p.ds_off = p.dx_off = p.part_off = at;
    if (grads) {
        at += align_up((size_t)p.slots * a.Hv * a.Dv * a.Dk * es, 256);
        p.dx_off = at;
        at += align_up((size_t)a.total * a.Hv * a.Dv * es, 256);
        p.part_off = at;
        if (grad_leaves_parts(a)) at += align_up((size_t)a.total * a.Hv * 2 * a.Dk * 4, 256);
    }
    p.bytes = at;
    return p;
}

vmb_status launch_delta_fwd(const DeltaArgs& a, cudaStream_t stream) {
    const DeltaPlan p = plan_delta(a, false, device_sm_count());
    if (a.ws_bytes < p.bytes) return VMB_ERR_WORKSPACE;
    DeltaChain c = chain_of(a, p);
    vmb_status s = clear(a, false, stream);
    if (s != VMB_OK) return s;
    if (p.segs > 1) {
        c.summary = 1;
        s = chain(c, false, stream);
        if (s == VMB_OK) s = join(c, false, stream);
        if (s != VMB_OK) return s;
        c.summary = 0;
    }
    return chain(c, false, stream);
}

vmb_status launch_delta_bwd(const DeltaArgs& a, cudaStream_t stream) {
    const DeltaPlan p = plan_delta(a, true, device_sm_count());
    if (a.ws_bytes < p.bytes) return VMB_ERR_WORKSPACE;
    DeltaChain c = chain_of(a, p);
    vmb_status s = clear(a, true, stream);
    if (s != VMB_OK) return s;
    if (p.segs > 1) {
        c.summary = c.maps_only = 1;
        if ((s = chain(c, false, stream)) != VMB_OK) return s;
        if ((s = chain(c, true, stream)) != VMB_OK) return s;
        if ((s = join(c, true, stream)) != VMB_OK) return s;
        c.summary = c.maps_only = 0;
    }
    if ((s = chain(c, true, stream)) != VMB_OK || a.T == 0 || a.total == 0) return s;
    DeltaGrad g{};
    g.a = a;
    g.ds = c.ds;
    g.dx = c.dx;
    g.part = (float*)((unsigned char*)a.ws + p.part_off);
    g.err = c.err;
    if ((s = a.dtype == VMB_BF16 ? launch_grad_bf16(g, stream) : launch_grad_f32(g, stream)) != VMB_OK) return s;
    if (!grad_leaves_parts(a)) return VMB_OK;
    void* args[] = {&g};
    return launch_kernel((const void*)delta_share_kernel, dim3((unsigned)((long long)a.B * chunks_of(a.T)), kShareCtas), dim3(256), 0, args, stream) ==
                   cudaSuccess ? VMB_OK : VMB_ERR_CUDA;
}

vmb_status launch_delta_step(const DeltaStep& a, cudaStream_t stream) {
    const long long grid = (long long)a.B * a.Hv * ((a.Dv + 63) / 64);
    const void* fn = a.dtype == VMB_BF16
                         ? (a.Dk <= 64 ? (const void*)delta_step_kernel<__nv_bfloat16, 8> : (const void*)delta_step_kernel<__nv_bfloat16, 16>)
                         : (a.Dk <= 64 ? (const void*)delta_step_kernel<float, 8> : (const void*)delta_step_kernel<float, 16>);
    DeltaStep arg = a;
    void* args[] = {&arg};
    return launch_kernel(fn, dim3((unsigned)grid), dim3(128), 0, args, stream) == cudaSuccess ? VMB_OK : VMB_ERR_CUDA;
}

}  // namespace vmb
