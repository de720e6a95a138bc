// delta_chain.cuh - the chains of the gated delta rule: the state carried from chunk to chunk
// (forward) and its gradient (reverse).  delta_common.cuh has the mathematics of a chunk.
//
// A CTA carries 64 rows (value channels) of one head's transposed state through the chunks of one
// segment, 16 rows per warp in registers, and computes the chunk's triangular system once for them.
// Chains too few to fill the GPU are cut into segments: the state after a segment is an affine map
// of the state before it, S' = M S + N, with N the state reached from zero and M the image of the
// identity with v = 0 (the same kernel, with Dk more rows).  A first launch computes M and N of
// every segment, delta_join_kernel (delta.cu) the state at every segment's start, a last launch the
// outputs.  The gradient of the state runs through M's transpose.
#pragma once

#include "delta_common.cuh"
#include "delta_internal.h"

namespace vmb {

template <typename T> struct DeltaTerms { static constexpr int mid = 2; };
template <> struct DeltaTerms<float> { static constexpr int mid = 1; };
__device__ __forceinline__ const FragA<__nv_bfloat16, 1>& lead(const FragA<__nv_bfloat16, 2>& a) {
    return reinterpret_cast<const FragA<__nv_bfloat16, 1>&>(a);
}
__device__ __forceinline__ const FragA<__nv_bfloat16, 1>& lead(const FragA<__nv_bfloat16, 1>& a) { return a; }
__device__ __forceinline__ const FragA<float, 1>& lead(const FragA<float, 1>& a) { return a; }

// Shared memory of the chain kernels, in bytes from the start.
template <typename T, int DK> struct ChainSmem {
    static constexpr int mid = DeltaTerms<T>::mid;
    using KT = Tile<T, DK, 1>;
    using VT = Tile<T, kDeltaRows, 1>;
    using ET = Tile<T, kChunk, mid>;
    using PT = Tile<T, kChunk, mid>;
    static constexpr int k = 0, q = k + KT::bytes(kChunk), v = q + KT::bytes(kChunk), stage = v + VT::bytes(kChunk);
    static constexpr int e = 2 * stage, p = e + ET::bytes(kChunk), diag = p + PT::bytes(kChunk),
                         gates = diag + 64 * 20 * 4, total = gates + (int)sizeof(ChunkGates);
};

// 16 x 64 (channel, token) accumulators of a warp to [token][channel] in global memory through the
// warp's 16 columns of a tile.
template <typename T>
__device__ __forceinline__ void store_tokens(const Tile<T, kDeltaRows, 1>& s, const float (&y)[8][4], T* dst, long long stride,
                                             int rows, int ch0, int channels, bool vec) {
    const int w = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    constexpr int V = Tile<T, kDeltaRows, 1>::kVec, P = 16 / V;
    __syncwarp();
#pragma unroll
    for (int n = 0; n < 8; ++n)
#pragma unroll
        for (int x = 0; x < 4; ++x) s.set(8 * n + 2 * t + (x & 1), 16 * w + g + 8 * (x >> 1), y[n][x]);
    __syncwarp();
    if (vec && ch0 + 16 * w + 16 <= channels) {
#pragma unroll
        for (int i = lane; i < kChunk * P; i += 32) {
            const int r = i / P, c = (i % P) * V;
            if (r < rows)
                *reinterpret_cast<uint4*>(dst + r * stride + ch0 + 16 * w + c) =
                    *reinterpret_cast<const uint4*>(s.vec_at(r, 16 * w + c));
        }
    } else {
        for (int i = lane; i < kChunk * 16; i += 32) {
            const int r = i >> 4, c = 16 * w + (i & 15);
            if (r < rows && ch0 + c < channels) dst[r * stride + ch0 + c] = *s.vec_at(r, c);
        }
    }
}

// A warp's 16 rows of the transposed state, [row][Dk] fp32 or storage type at dst.
template <int DK, typename T>
__device__ __forceinline__ void store_state_rows(const float (&S)[DK / 8][4], T* dst, int row0, int rows, int Dk) {
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int r = row0 + g + 8 * h;
        if (r >= rows) continue;
        T* p = dst + (long long)r * Dk;
#pragma unroll
        for (int n = 0; n < DK / 8; ++n) {
            const int d = 8 * n + 2 * t;
            if (d < Dk) p[d] = io<T>::to(S[n][2 * h]);
            if (d + 1 < Dk) p[d + 1] = io<T>::to(S[n][2 * h + 1]);
        }
    }
}
template <int DK>
__device__ __forceinline__ void load_state_rows(float (&S)[DK / 8][4], const float* src, int row0, int rows, int Dk, int row_step,
                                                int col_step) {
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
#pragma unroll
    for (int n = 0; n < DK / 8; ++n)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const int r = row0 + g + 8 * (x >> 1), d = 8 * n + 2 * t + (x & 1);
            S[n][x] = r < rows && d < Dk ? src[(long long)r * row_step + (long long)d * col_step] : 0.0f;
        }
}

// Where a CTA works: chain, segment, slice of rows.
struct ChainPlace {
    int b, h, seg, slice;
    long long chain;
};
__device__ __forceinline__ ChainPlace chain_place(const DeltaChain& c, int slices) {
    ChainPlace p;
    const unsigned i = blockIdx.x, rest = i / slices;
    p.slice = i % slices;
    p.seg = rest % c.segs;
    p.chain = rest / c.segs;
    p.h = (int)(p.chain % c.a.Hv);
    p.b = (int)(p.chain / c.a.Hv);
    return p;
}

// The two tokens of lane l of a warp: g and beta, zeros behind the end.
template <typename T>
__device__ __forceinline__ void load_gates(const T* g, const T* beta, int rows, int Hv, float (&v)[4]) {
    const int i = 2 * (threadIdx.x & 31);
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        v[x] = i + x < rows ? io<T>::cvt(g[(long long)(i + x) * Hv]) : 0.0f;
        v[2 + x] = i + x < rows ? io<T>::cvt(beta[(long long)(i + x) * Hv]) : 0.0f;
    }
}

// kOut = false: the maps and sums of a segment (DeltaChain::summary).
template <typename T, int DK, bool kOut>
__global__ void __launch_bounds__(kDeltaThreads) delta_forward_kernel(DeltaChain c) {
    using SM = ChainSmem<T, DK>;
    constexpr int M = SM::mid;
    extern __shared__ __align__(128) unsigned char smem[];
    const DeltaArgs& a = c.a;
    const int w = threadIdx.x >> 5, t = threadIdx.x & 3;
    pdl_launch_dependents();
    pdl_wait();
    const int vslices = c.slices, mslices = kOut ? 0 : (a.Dk + kDeltaRows - 1) / kDeltaRows;
    ChainPlace at = chain_place(c, kOut ? vslices : (c.maps_only ? mslices : vslices + mslices));
    const bool map = !kOut && (c.maps_only || at.slice >= vslices);  // rows of the map: v = 0, S = identity
    const int slice = map && !c.maps_only ? at.slice - vslices : at.slice;
    const DeltaSeq seq = delta_seq(a.offsets, at.b, a.T, a.total, c.err);
    const int nc = (seq.len + kChunk - 1) / kChunk;
    const int c0 = at.seg * c.seg_chunks, c1 = min(nc, c0 + c.seg_chunks);
    const int row0 = slice * kDeltaRows + 16 * w, rows = map ? a.Dk : a.Dv;

    float S[DK / 8][4];
    if (kOut && c.segs > 1) {
        if (c0 >= nc) return;
        load_state_rows<DK>(S, c.sums + (at.chain * c.segs + at.seg) * a.Dv * a.Dk, row0, rows, a.Dk, a.Dk, 1);
    } else if (kOut && a.initial) {
        load_state_rows<DK>(S, a.initial + at.chain * a.Dk * a.Dv, row0, rows, a.Dk, 1, a.Dv);
    } else {
        const int g = (threadIdx.x & 31) >> 2;
#pragma unroll
        for (int n = 0; n < DK / 8; ++n)
#pragma unroll
            for (int x = 0; x < 4; ++x)
                S[n][x] = map && row0 + g + 8 * (x >> 1) == 8 * n + 2 * t + (x & 1) ? 1.0f : 0.0f;
    }
    if (!kOut && c0 >= nc) return;

    const int hk = at.h / (a.Hv / a.Hk);
    const long long brow = a.offsets ? 0 : at.b, tok0 = a.offsets ? seq.start : 0;
    const T* kp = (const T*)a.k + brow * a.k_b + tok0 * a.k_t + (long long)hk * a.Dk;
    const T* qp = (const T*)a.q + brow * a.q_b + tok0 * a.q_t + (long long)hk * a.Dk;
    const T* vp = (const T*)a.v + brow * a.v_b + tok0 * a.v_t + (long long)at.h * a.Dv + slice * kDeltaRows;
    const T* gp = (const T*)a.g + seq.start * a.Hv + at.h;
    const T* bp = (const T*)a.beta + seq.start * a.Hv + at.h;
    T* op = kOut ? (T*)a.o + (seq.start * a.Hv + at.h) * a.Dv : nullptr;
    const bool kvec = rows_aligned(kp, a.k_t), qvec = rows_aligned(qp, a.q_t), vvec = rows_aligned(vp, a.v_t);
    T* rp = kOut && a.saved_r ? (T*)a.saved_r + (seq.start * a.Hv + at.h) * a.Dv : nullptr;
    const bool rvec = kOut && rows_aligned(rp, (long long)a.Hv * a.Dv);
    const bool ovec = kOut && rows_aligned(op, (long long)a.Hv * a.Dv);
    const int vcols = min(a.Dv - slice * kDeltaRows, kDeltaRows);

    const typename SM::ET sE(smem + SM::e, kChunk);
    const typename SM::PT sP(smem + SM::p, kChunk);
    float* diag = reinterpret_cast<float*>(smem + SM::diag);
    ChunkGates& G = *reinterpret_cast<ChunkGates*>(smem + SM::gates);
    float gv[4];

    auto load = [&](int ch) {
        unsigned char* s = smem + (ch & 1) * SM::stage;
        const long long t0 = (long long)ch * kChunk;
        const int n = min(seq.len - ch * kChunk, kChunk);
        load_tile<kChunk, DK>(typename SM::KT(s + SM::k, kChunk), kp + t0 * a.k_t, a.k_t, n, a.Dk, kvec, threadIdx.x, kDeltaThreads);
        if (kOut)
            load_tile<kChunk, DK>(typename SM::KT(s + SM::q, kChunk), qp + t0 * a.q_t, a.q_t, n, a.Dk, qvec, threadIdx.x, kDeltaThreads);
        if (!map)
            load_tile<kChunk, kDeltaRows>(typename SM::VT(s + SM::v, kChunk), vp + t0 * a.v_t, a.v_t, n, vcols, vvec, threadIdx.x, kDeltaThreads);
        cp_async_commit();
        if (w == 0) load_gates(gp + t0 * a.Hv, bp + t0 * a.Hv, n, a.Hv, gv);
    };
    if (c0 < c1) load(c0);
    for (int ch = c0; ch < c1; ++ch) {
        unsigned char* s = smem + (ch & 1) * SM::stage;
        const typename SM::KT sK(s + SM::k, kChunk), sQ(s + SM::q, kChunk);
        const typename SM::VT sV(s + SM::v, kChunk);
        if (w == 0) chunk_gates(G, gv[0], gv[1], gv[2], gv[3]);
        if (ch + 1 < c1) load(ch + 1);
        if (ch + 1 < c1) cp_async_wait<1>(); else cp_async_wait<0>();
        __syncthreads();
        chunk_system<T, DK, false, kOut>(sK, sQ, sE, sP, diag, G, a.scale, kDeltaThreads / 32);
        if (kOut && a.saved)
            store_state_rows<DK>(S, (T*)a.saved + ((long long)(seq.slot + ch) * a.Hv + at.h) * a.Dv * a.Dk, row0, a.Dv, a.Dk);

        float x[8][4] = {}, y[kOut ? 8 : 1][4] = {};  // K S and Q S, transposed: [channel][token]
#pragma unroll
        for (int d = 0; d < DK / 16; ++d) {
            FragA<T, M> f;
            frag_from_acc(f, S[2 * d], S[2 * d + 1]);
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                FragB<T, 1> b0, b1;
                sK.b_nk(b0, b1, 16 * n, 16 * d);
                mma16(x[2 * n], f, b0);
                mma16(x[2 * n + 1], f, b1);
                if constexpr (kOut) {
                    sQ.b_nk(b0, b1, 16 * n, 16 * d);
                    mma16(y[2 * n], lead(f), b0);
                    mma16(y[2 * n + 1], lead(f), b1);
                }
            }
        }
#pragma unroll
        for (int n = 0; n < DK / 8; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) S[n][i] *= G.last;
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            float v0[4] = {}, v1[4] = {};
            if (!map) sV.acc_km(v0, v1, 16 * w, 16 * n);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float e0 = G.ec[16 * n + 2 * t + (i & 1)], e1 = G.ec[16 * n + 8 + 2 * t + (i & 1)];
                x[2 * n][i] = v0[i] - e0 * x[2 * n][i];
                x[2 * n + 1][i] = v1[i] - e1 * x[2 * n + 1][i];
                if constexpr (kOut) {
                    y[2 * n][i] *= a.scale * e0;
                    y[2 * n + 1][i] *= a.scale * e1;
                }
            }
        }
        FragA<T, M> uf[4];
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            float r0[4] = {}, r1[4] = {};
            FragB<T, M> e0, e1;
#pragma unroll
            for (int j = 0; j < b; ++j) {
                sE.b_nk(e0, e1, 16 * b, 16 * j);
                mma16(x[2 * b], uf[j], e0);
                mma16(x[2 * b + 1], uf[j], e1);
            }
            FragA<T, M> f;
            frag_from_acc(f, x[2 * b], x[2 * b + 1]);
            sE.b_nk(e0, e1, 16 * b, 16 * b);
            mma16(r0, f, e0);
            mma16(r1, f, e1);
            if constexpr (kOut) {
#pragma unroll
                for (int i = 0; i < 4; ++i) x[2 * b][i] = r0[i], x[2 * b + 1][i] = r1[i];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                r0[i] *= G.beta[16 * b + 2 * t + (i & 1)];
                r1[i] *= G.beta[16 * b + 8 + 2 * t + (i & 1)];
            }
            frag_from_acc(uf[b], r0, r1);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                r0[i] *= G.tail[16 * b + 2 * t + (i & 1)];
                r1[i] *= G.tail[16 * b + 8 + 2 * t + (i & 1)];
            }
            frag_from_acc(f, r0, r1);
#pragma unroll
            for (int d = 0; d < DK / 16; ++d) {
                FragB<T, 1> k0, k1;
                sK.b_kn(k0, k1, 16 * b, 16 * d);
                mma16(S[2 * d], f, k0);
                mma16(S[2 * d + 1], f, k1);
            }
            if constexpr (kOut) {
#pragma unroll
                for (int n = b; n < 4; ++n) {
                    FragB<T, M> p0, p1;
                    sP.b_nk(p0, p1, 16 * n, 16 * b);
                    mma16(y[2 * n], uf[b], p0);
                    mma16(y[2 * n + 1], uf[b], p1);
                }
            }
        }
        if constexpr (kOut) {
            const long long hrow = (long long)a.Hv * a.Dv, at0 = (long long)ch * kChunk * hrow;
            const int n = min(seq.len - ch * kChunk, kChunk);
            store_tokens<T>(sV, y, op + at0, hrow, n, slice * kDeltaRows, a.Dv, ovec);
            if (rp) store_tokens<T>(sV, x, rp + at0, hrow, n, slice * kDeltaRows, a.Dv, rvec);
        }
        __syncthreads();  // the tiles of this chunk are rewritten two loads from here
    }
    if constexpr (kOut) {
        if (a.final && c.segs == 1) {
            const int g = (threadIdx.x & 31) >> 2;
            float* dst = a.final + at.chain * a.Dk * a.Dv;
#pragma unroll
            for (int n = 0; n < DK / 8; ++n)
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const int r = row0 + g + 8 * (x >> 1), d = 8 * n + 2 * t + (x & 1);
                    if (r < a.Dv && d < a.Dk) dst[(long long)d * a.Dv + r] = S[n][x];
                }
        }
    } else {
        const long long i = at.chain * c.segs + at.seg;
        if (map)
            store_state_rows<DK>(S, c.maps + i * a.Dk * a.Dk, row0, a.Dk, a.Dk);
        else
            store_state_rows<DK>(S, c.sums + i * a.Dv * a.Dk, row0, a.Dv, a.Dk);
    }
}

// The reverse: dS (transposed, like S) from the last chunk to the first,
//   dU = P^T do + tail K dS,  dX = (I + b E)^-T dU,  dR = b dX,
//   dS <- e^(c_last) dS + (scale e^c Q)^T do - (e^c K)^T dR.
// Writes dS at each chunk's end, dX and dv = dR of every token; with DeltaChain::summary only the segment's sum.
template <typename T, int DK>
__global__ void __launch_bounds__(kDeltaThreads) delta_reverse_kernel(DeltaChain c) {
    using SM = ChainSmem<T, DK>;
    constexpr int M = SM::mid;
    extern __shared__ __align__(128) unsigned char smem[];
    const DeltaArgs& a = c.a;
    const int w = threadIdx.x >> 5, t = threadIdx.x & 3, g = (threadIdx.x & 31) >> 2;
    pdl_launch_dependents();
    pdl_wait();
    const ChainPlace at = chain_place(c, c.slices);
    const DeltaSeq seq = delta_seq(a.offsets, at.b, a.T, a.total, c.err);
    const int nc = (seq.len + kChunk - 1) / kChunk;
    const int c0 = at.seg * c.seg_chunks, c1 = min(nc, c0 + c.seg_chunks);
    const int row0 = at.slice * kDeltaRows + 16 * w;

    float S[DK / 8][4];
    if (c.segs > 1 && c0 >= nc) return;
    if (!c.summary && c.segs > 1) {
        load_state_rows<DK>(S, c.sums + (at.chain * c.segs + at.seg) * a.Dv * a.Dk, row0, a.Dv, a.Dk, a.Dk, 1);
    } else if (!c.summary && a.dfinal) {
        load_state_rows<DK>(S, a.dfinal + at.chain * a.Dk * a.Dv, row0, a.Dv, a.Dk, 1, a.Dv);
    } else {
#pragma unroll
        for (int n = 0; n < DK / 8; ++n)
#pragma unroll
            for (int x = 0; x < 4; ++x) S[n][x] = 0.0f;
    }

    const int hk = at.h / (a.Hv / a.Hk);
    const long long brow = a.offsets ? 0 : at.b, tok0 = a.offsets ? seq.start : 0;
    const T* kp = (const T*)a.k + brow * a.k_b + tok0 * a.k_t + (long long)hk * a.Dk;
    const T* qp = (const T*)a.q + brow * a.q_b + tok0 * a.q_t + (long long)hk * a.Dk;
    const long long hrow = (long long)a.Hv * a.Dv;  // do and dX are dense
    const T* dp = (const T*)a.dout + seq.start * hrow + (long long)at.h * a.Dv + at.slice * kDeltaRows;
    T* xp = (T*)c.dx + seq.start * hrow + (long long)at.h * a.Dv;
    const T* gp = (const T*)a.g + seq.start * a.Hv + at.h;
    const T* bp = (const T*)a.beta + seq.start * a.Hv + at.h;
    const bool kvec = rows_aligned(kp, a.k_t), qvec = rows_aligned(qp, a.q_t), dvec = rows_aligned(dp, hrow);
    T* rp = (T*)a.dv + seq.start * hrow + (long long)at.h * a.Dv;
    const bool xvec = rows_aligned(xp, hrow), rvec = rows_aligned(rp, hrow);
    const int vcols = min(a.Dv - at.slice * kDeltaRows, kDeltaRows);

    const typename SM::ET sE(smem + SM::e, kChunk);
    const typename SM::PT sP(smem + SM::p, kChunk);
    float* diag = reinterpret_cast<float*>(smem + SM::diag);
    ChunkGates& G = *reinterpret_cast<ChunkGates*>(smem + SM::gates);
    float gv[4];

    auto load = [&](int ch) {
        unsigned char* s = smem + (ch & 1) * SM::stage;
        const long long t0 = (long long)ch * kChunk;
        const int n = min(seq.len - ch * kChunk, kChunk);
        load_tile<kChunk, DK>(typename SM::KT(s + SM::k, kChunk), kp + t0 * a.k_t, a.k_t, n, a.Dk, kvec, threadIdx.x, kDeltaThreads);
        load_tile<kChunk, DK>(typename SM::KT(s + SM::q, kChunk), qp + t0 * a.q_t, a.q_t, n, a.Dk, qvec, threadIdx.x, kDeltaThreads);
        load_tile<kChunk, kDeltaRows>(typename SM::VT(s + SM::v, kChunk), dp + t0 * hrow, hrow, n, vcols, dvec, threadIdx.x, kDeltaThreads);
        cp_async_commit();
        if (w == 0) load_gates(gp + t0 * a.Hv, bp + t0 * a.Hv, n, a.Hv, gv);
    };
    if (c0 < c1) load(c1 - 1);
    for (int ch = c1 - 1; ch >= c0; --ch) {
        unsigned char* s = smem + (ch & 1) * SM::stage;
        const typename SM::KT sK(s + SM::k, kChunk), sQ(s + SM::q, kChunk);
        const typename SM::VT sD(s + SM::v, kChunk);
        if (w == 0) chunk_gates(G, gv[0], gv[1], gv[2], gv[3]);
        if (ch > c0) load(ch - 1);
        if (ch > c0) cp_async_wait<1>(); else cp_async_wait<0>();
        __syncthreads();
        chunk_system<T, DK, true, true>(sK, sQ, sE, sP, diag, G, a.scale, kDeltaThreads / 32);
        if (!c.summary)
            store_state_rows<DK>(S, (T*)c.ds + ((long long)(seq.slot + ch) * a.Hv + at.h) * a.Dv * a.Dk, row0, a.Dv, a.Dk);

        float x[8][4] = {};  // dU, then dX, transposed
#pragma unroll
        for (int d = 0; d < DK / 16; ++d) {
            FragA<T, M> f;
            frag_from_acc(f, S[2 * d], S[2 * d + 1]);
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                FragB<T, 1> b0, b1;
                sK.b_nk(b0, b1, 16 * n, 16 * d);
                mma16(x[2 * n], f, b0);
                mma16(x[2 * n + 1], f, b1);
            }
        }
#pragma unroll
        for (int n = 0; n < DK / 8; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) S[n][i] *= G.last;
#pragma unroll
        for (int n = 0; n < 8; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) x[n][i] *= G.tail[8 * n + 2 * t + (i & 1)];
#pragma unroll
        for (int b = 0; b < 4; ++b) {  // token block b of do: P^T do into dU, (scale e^c Q)^T do into dS
            FragA<T, 1> f;
            sD.a_km(f, 16 * w, 16 * b);
#pragma unroll
            for (int n = 0; n <= b; ++n) {
                FragB<T, M> p0, p1;
                sP.b_kn(p0, p1, 16 * b, 16 * n);
                mma16(x[2 * n], f, p0);
                mma16(x[2 * n + 1], f, p1);
            }
            float d0[4], d1[4];
            sD.acc_km(d0, d1, 16 * w, 16 * b);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                d0[i] *= a.scale * G.ec[16 * b + 2 * t + (i & 1)];
                d1[i] *= a.scale * G.ec[16 * b + 8 + 2 * t + (i & 1)];
            }
            FragA<T, M> fs;
            frag_from_acc(fs, d0, d1);
#pragma unroll
            for (int d = 0; d < DK / 16; ++d) {
                FragB<T, 1> q0, q1;
                sQ.b_kn(q0, q1, 16 * b, 16 * d);
                mma16(S[2 * d], fs, q0);
                mma16(S[2 * d + 1], fs, q1);
            }
        }
        FragA<T, M> rf[4];
#pragma unroll
        for (int b = 3; b >= 0; --b) {
            FragB<T, M> e0, e1;
#pragma unroll
            for (int j = 3; j > b; --j) {
                sE.b_kn(e0, e1, 16 * j, 16 * b);
                mma16(x[2 * b], rf[j], e0);
                mma16(x[2 * b + 1], rf[j], e1);
            }
            FragA<T, M> f;
            frag_from_acc(f, x[2 * b], x[2 * b + 1]);
            float r0[4] = {}, r1[4] = {};
            sE.b_kn(e0, e1, 16 * b, 16 * b);
            mma16(r0, f, e0);
            mma16(r1, f, e1);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[2 * b][i] = r0[i];
                x[2 * b + 1][i] = r1[i];
                r0[i] *= G.beta[16 * b + 2 * t + (i & 1)];
                r1[i] *= G.beta[16 * b + 8 + 2 * t + (i & 1)];
            }
            frag_from_acc(rf[b], r0, r1);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                r0[i] *= -G.ec[16 * b + 2 * t + (i & 1)];
                r1[i] *= -G.ec[16 * b + 8 + 2 * t + (i & 1)];
            }
            frag_from_acc(f, r0, r1);
#pragma unroll
            for (int d = 0; d < DK / 16; ++d) {
                FragB<T, 1> k0, k1;
                sK.b_kn(k0, k1, 16 * b, 16 * d);
                mma16(S[2 * d], f, k0);
                mma16(S[2 * d + 1], f, k1);
            }
        }
        if (!c.summary) {
            const int n = min(seq.len - ch * kChunk, kChunk);
            store_tokens<T>(sD, x, xp + (long long)ch * kChunk * hrow, hrow, n, at.slice * kDeltaRows, a.Dv, xvec);
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) x[i][j] *= G.beta[8 * i + 2 * t + (j & 1)];
            store_tokens<T>(sD, x, rp + (long long)ch * kChunk * hrow, hrow, n, at.slice * kDeltaRows, a.Dv, rvec);
        }
        __syncthreads();
    }
    if (c.summary) {
        store_state_rows<DK>(S, c.sums + (at.chain * c.segs + at.seg) * a.Dv * a.Dk, row0, a.Dv, a.Dk);
    } else if (a.dinitial && c.segs == 1) {
        float* dst = a.dinitial + at.chain * a.Dk * a.Dv;
#pragma unroll
        for (int n = 0; n < DK / 8; ++n)
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int r = row0 + g + 8 * (x >> 1), d = 8 * n + 2 * t + (x & 1);
                if (r < a.Dv && d < a.Dk) dst[(long long)d * a.Dv + r] = S[n][x];
            }
    }
}

template <typename T, int DK>
vmb_status launch_chain_dk(const DeltaChain& c, bool reverse, cudaStream_t stream) {
    const void* fn = reverse ? (const void*)delta_reverse_kernel<T, DK>
                             : c.summary ? (const void*)delta_forward_kernel<T, DK, false> : (const void*)delta_forward_kernel<T, DK, true>;
    const int mslices = (c.a.Dk + kDeltaRows - 1) / kDeltaRows;
    const long long per = reverse || !c.summary ? c.slices : c.maps_only ? mslices : c.slices + mslices;
    const long long grid = (long long)c.a.B * c.a.Hv * c.segs * per;
    const size_t smem = ChainSmem<T, DK>::total;
    if (cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) return VMB_ERR_CUDA;
    DeltaChain arg = c;
    void* args[] = {&arg};
    return launch_kernel(fn, dim3((unsigned)grid), dim3(kDeltaThreads), smem, args, stream) == cudaSuccess ? VMB_OK : VMB_ERR_CUDA;
}

template <typename T>
vmb_status launch_chain(const DeltaChain& c, bool reverse, cudaStream_t stream) {
    return c.a.Dk <= 64 ? launch_chain_dk<T, 64>(c, reverse, stream) : launch_chain_dk<T, 128>(c, reverse, stream);
}

}  // namespace vmb
