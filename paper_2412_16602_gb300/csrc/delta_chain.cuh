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

// Roles: warps 0 to 3 carry the state (240 registers), warps 4 to 11 load the tiles of the chunks ahead and compute
// their triangular systems (128 registers; 128 x 240 + 256 x 128 is within the 384 x 168 of the launch).  Done one
// after the other by four warps, loads and system took 8400 of a chunk's 14400 cycles (bf16, Dk = 64).
constexpr int kChainThreads = 384, kStateThreads = 128, kSystemThreads = 256;
constexpr int kBarSystem = 1, kBarFull = 2, kBarEmpty = 4;  // named barriers; full and empty: + parity of the chunk
__device__ __forceinline__ void bar_sync(int id, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }
__device__ __forceinline__ void bar_arrive(int id, int threads) { asm volatile("bar.arrive %0, %1;" ::"r"(id), "r"(threads) : "memory"); }

// Shared memory of the chain kernels, in bytes from the start: a ring of tiles, two systems.
template <typename T, int DK> struct ChainSmem {
    static constexpr int mid = DeltaTerms<T>::mid;
    using KT = Tile<T, DK, 1>;
    using VT = Tile<T, kDeltaRows, 1>;
    using ET = LowTile<T, mid>;
    static constexpr int ring = sizeof(T) == 4 && DK == 128 ? 2 : 3;
    static constexpr int k = 0, q = k + KT::bytes(kChunk), v = q + KT::bytes(kChunk), stage = v + VT::bytes(kChunk);
    static constexpr int e = 0, p = e + ET::kBytes, system = p + ET::kBytes;
    static constexpr int gate = (sizeof(ChunkGates) + 15) & ~15;  // three of them: a chunk's are computed ahead
    static constexpr int systems = ring * stage, diag = systems + 2 * system, gates = diag + 64 * 20 * 4, total = gates + 3 * gate;
    static_assert(total <= 227 * 1024 && system % 16 == 0 && stage % 16 == 0, "fits");
};

// 16 x 64 (channel, token) accumulators of a warp to [token][channel] in global memory through the
// warp's 16 columns of a tile.
template <typename T>
__device__ __forceinline__ void store_tokens(const Tile<T, kDeltaRows, 1>& s, const float (&y)[8][4], T* dst, long long stride,
                                             int rows, int ch0, int channels, bool vec) {
    const int w = threadIdx.x >> 5, lane = threadIdx.x & 31;
    constexpr int V = Tile<T, kDeltaRows, 1>::kVec, P = 16 / V;
    __syncwarp();
#pragma unroll
    for (int n = 0; n < 4; ++n) s.set_t(16 * n, 16 * w, y[2 * n], y[2 * n + 1]);
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

// The loads and systems of the chunks of a chain, first to last (step = 1) or last to first, by the system warps.
// `tiles` loads a chunk's tiles into a stage; `gates` gives the two tokens' g and beta of a lane.
template <typename T, int DK, bool kRowBeta, bool kWithP, typename Tiles, typename Gates>
__device__ __forceinline__ void system_warps(unsigned char* smem, int chunks, float scale, Tiles tiles, Gates gates) {
    using SM = ChainSmem<T, DK>;
    constexpr int kGateWarp = 7;  // has one block of the system, others up to two or an inverse
    const int tid = threadIdx.x - kStateThreads, w = tid >> 5;
    float* diag = reinterpret_cast<float*>(smem + SM::diag);
    auto gate = [&](int i) -> ChunkGates& { return *reinterpret_cast<ChunkGates*>(smem + SM::gates + (i % 3) * SM::gate); };
    float gv[4];
    constexpr bool kAhead = SM::ring == 3;
    if (kAhead && chunks > 0) {
        tiles(0, smem, tid);
        cp_async_commit();
    }
    if (w == kGateWarp && chunks > 0) {
        gates(0, gv);
        chunk_gates(gate(0), gv[0], gv[1], gv[2], gv[3]);
        if (chunks > 1) gates(1, gv);
    }
    for (int i = 0; i < chunks; ++i) {
        // the states are done with chunk i - 2: its system, and with it the oldest stage and gates, are free
        if (i >= 2) bar_sync(kBarEmpty + (i & 1), kChainThreads);
        if (kAhead ? i + 1 < chunks : true) {
            const int next = kAhead ? i + 1 : i;
            tiles(next, smem + (next % SM::ring) * SM::stage, tid);
            cp_async_commit();
        }
        unsigned char *st = smem + (i % SM::ring) * SM::stage, *sy = smem + SM::systems + (i & 1) * SM::system;
        if (kAhead && i + 1 < chunks) cp_async_wait<1>(); else cp_async_wait<0>();
        bar_sync(kBarSystem, kSystemThreads);
        chunk_system<T, DK, kRowBeta, kWithP>(typename SM::KT(st + SM::k, kChunk), typename SM::KT(st + SM::q, kChunk),
                                              typename SM::ET(sy + SM::e), typename SM::ET(sy + SM::p), diag, gate(i), scale, w);
        if (w == kGateWarp && i + 1 < chunks) {
            chunk_gates(gate(i + 1), gv[0], gv[1], gv[2], gv[3]);
            if (i + 2 < chunks) gates(i + 2, gv);
        }
        bar_arrive(kBarFull + (i & 1), kChainThreads);
    }
    // the last two releases, so that every barrier is left complete
    for (int i = chunks < 2 ? 0 : chunks - 2; i < chunks; ++i) bar_sync(kBarEmpty + (i & 1), kChainThreads);
}

// x[channel][token] += S^T K^T and, with kTwo, y += S^T Q^T (leading terms of S), the rows of the state against every
// token; the operands of the next four tiles are read before the products of these.
template <int DK, bool kTwo, int NS, typename T, typename TL>
__device__ __forceinline__ void state_times(const float (&S)[DK / 8][4], float (&x)[8][4], float (*y)[4], const TL& sK, const TL& sQ) {
    constexpr int kSteps = DK / 16 * (kTwo ? 4 : 2);
    FragB<T, 1> b[2][4];
    auto read = [&](int i, FragB<T, 1>(&f)[4]) {
        const int d = kTwo ? i >> 2 : i >> 1, n = 32 * (kTwo ? (i >> 1) & 1 : i & 1);
        const TL& s = kTwo && (i & 1) ? sQ : sK;
        s.b_nk(f[0], f[1], n, 16 * d);
        s.b_nk(f[2], f[3], n + 16, 16 * d);
    };
    read(0, b[0]);
    FragA<T, NS> f;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        if (i + 1 < kSteps) read(i + 1, b[(i + 1) & 1]);
        const int d = kTwo ? i >> 2 : i >> 1, n = 4 * (kTwo ? (i >> 1) & 1 : i & 1);
        if (kTwo ? i % 4 == 0 : i % 2 == 0) frag_from_acc(f, S[2 * d], S[2 * d + 1]);
        if (kTwo && (i & 1))
            mma_quad(*reinterpret_cast<float(*)[4][4]>(&y[n]), lead(f), b[i & 1]);
        else
            mma_quad(*reinterpret_cast<float(*)[4][4]>(&x[n]), f, b[i & 1]);
    }
}
// S += f K_b: the outer products of 16 tokens (block b of a tile) with the state's columns
template <int DK, int NS, typename T, typename TL>
__device__ __forceinline__ void state_add(float (&S)[DK / 8][4], const FragA<T, NS>& f, const TL& s, int b) {
#pragma unroll
    for (int d = 0; d < DK / 32; ++d) {
        FragB<T, 1> k[4];
        s.b_kn(k[0], k[1], 16 * b, 32 * d);
        s.b_kn(k[2], k[3], 16 * b, 32 * d + 16);
        mma_quad(*reinterpret_cast<float(*)[4][4]>(&S[4 * d]), f, k);
    }
}

// kOut = false: the maps and sums of a segment (DeltaChain::summary).
template <typename T, int DK, bool kOut>
__global__ void __launch_bounds__(kChainThreads, 1) delta_forward_kernel(DeltaChain c) {
    using SM = ChainSmem<T, DK>;
    constexpr int M = SM::mid;
    extern __shared__ __align__(128) unsigned char smem[];
    const DeltaArgs& a = c.a;
    pdl_launch_dependents();
    pdl_wait();
    const int vslices = c.slices, mslices = kOut ? 0 : (a.Dk + kDeltaRows - 1) / kDeltaRows;
    const ChainPlace at = chain_place(c, kOut ? vslices : (c.maps_only ? mslices : vslices + mslices));
    const bool map = !kOut && (c.maps_only || at.slice >= vslices);  // rows of the map: v = 0, S = identity
    const int slice = map && !c.maps_only ? at.slice - vslices : at.slice;
    const DeltaSeq seq = delta_seq(a.offsets, at.b, a.T, a.total, c.err);
    const int nc = (seq.len + kChunk - 1) / kChunk;
    const int c0 = at.seg * c.seg_chunks, c1 = min(nc, c0 + c.seg_chunks);
    if ((!kOut || c.segs > 1) && c0 >= nc) return;
    const long long hrow = (long long)a.Hv * a.Dv;

    if (threadIdx.x >= kStateThreads) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 128;");
        const int hk = at.h / (a.Hv / a.Hk);
        const long long brow = a.offsets ? 0 : at.b, tok0 = a.offsets ? seq.start : 0;
        const T* kp = (const T*)a.k + brow * a.k_b + tok0 * a.k_t + (long long)hk * a.Dk;
        const T* qp = (const T*)a.q + brow * a.q_b + tok0 * a.q_t + (long long)hk * a.Dk;
        const T* vp = (const T*)a.v + brow * a.v_b + tok0 * a.v_t + (long long)at.h * a.Dv + slice * kDeltaRows;
        const T* gp = (const T*)a.g + seq.start * a.Hv + at.h;
        const T* bp = (const T*)a.beta + seq.start * a.Hv + at.h;
        const int ptid = threadIdx.x - kStateThreads;
        const TileCopy<typename SM::KT, DK, kSystemThreads> ck(kp, a.k_t, a.Dk, ptid), cq(qp, a.q_t, a.Dk, ptid);
        const TileCopy<typename SM::VT, kDeltaRows, kSystemThreads> cv(vp, a.v_t, min(a.Dv - slice * kDeltaRows, kDeltaRows), ptid);
        system_warps<T, DK, false, kOut>(
            smem, c1 - c0, a.scale,
            [&](int i, unsigned char* s, int tid) {
                const int first = (c0 + i) * kChunk, n = min(seq.len - first, kChunk);
                ck.copy(s + SM::k, first, n, tid);
                if (kOut) cq.copy(s + SM::q, first, n, tid);
                if (!map) cv.copy(s + SM::v, first, n, tid);
            },
            [&](int i, float(&v)[4]) {
                const long long t0 = (long long)(c0 + i) * kChunk * a.Hv;
                load_gates(gp + t0, bp + t0, min(seq.len - (c0 + i) * kChunk, kChunk), a.Hv, v);
            });
        return;
    }
    asm volatile("setmaxnreg.inc.sync.aligned.u32 240;");
    const int w = threadIdx.x >> 5, t = threadIdx.x & 3, g = (threadIdx.x & 31) >> 2;
    const int row0 = slice * kDeltaRows + 16 * w;
    T* op = kOut ? (T*)a.o + seq.start * hrow + (long long)at.h * a.Dv : nullptr;
    T* rp = kOut && a.saved_r ? (T*)a.saved_r + seq.start * hrow + (long long)at.h * a.Dv : nullptr;
    const bool ovec = kOut && rows_aligned(op, hrow), rvec = kOut && rows_aligned(rp, hrow);

    float S[DK / 8][4];
    if (kOut && c.segs > 1) {
        load_state_rows<DK>(S, c.sums + (at.chain * c.segs + at.seg) * a.Dv * a.Dk, row0, a.Dv, a.Dk, a.Dk, 1);
    } else if (kOut && a.initial) {
        load_state_rows<DK>(S, a.initial + at.chain * a.Dk * a.Dv, row0, a.Dv, a.Dk, 1, a.Dv);
    } else {
#pragma unroll
        for (int n = 0; n < DK / 8; ++n)
#pragma unroll
            for (int x = 0; x < 4; ++x)
                S[n][x] = map && row0 + g + 8 * (x >> 1) == 8 * n + 2 * t + (x & 1) ? 1.0f : 0.0f;
    }

    for (int i = 0; i < c1 - c0; ++i) {
        const int ch = c0 + i;
        unsigned char *st = smem + (i % SM::ring) * SM::stage, *sy = smem + SM::systems + (i & 1) * SM::system;
        const typename SM::KT sK(st + SM::k, kChunk), sQ(st + SM::q, kChunk);
        const typename SM::VT sV(st + SM::v, kChunk);
        const typename SM::ET sE(sy + SM::e), sP(sy + SM::p);
        const ChunkGates& G = *reinterpret_cast<const ChunkGates*>(smem + SM::gates + (i % 3) * SM::gate);
        bar_sync(kBarFull + (i & 1), kChainThreads);
        if (kOut && a.saved)
            store_state_rows<DK>(S, (T*)a.saved + ((long long)(seq.slot + ch) * a.Hv + at.h) * a.Dv * a.Dk, row0, a.Dv, a.Dk);

        float x[8][4] = {}, y[kOut ? 8 : 1][4] = {};  // K S and Q S, transposed: [channel][token]
        state_times<DK, kOut, M, T>(S, x, y, sK, sQ);
#pragma unroll
        for (int n = 0; n < DK / 8; ++n)
#pragma unroll
            for (int j = 0; j < 4; ++j) S[n][j] *= G.last;
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            float v0[4] = {}, v1[4] = {};
            if (!map) sV.acc_km(v0, v1, 16 * w, 16 * n);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float e0 = G.ec[16 * n + 2 * t + (j & 1)], e1 = G.ec[16 * n + 8 + 2 * t + (j & 1)];
                x[2 * n][j] = v0[j] - e0 * x[2 * n][j];
                x[2 * n + 1][j] = v1[j] - e1 * x[2 * n + 1][j];
                if constexpr (kOut) {
                    y[2 * n][j] *= a.scale * e0;
                    y[2 * n + 1][j] *= a.scale * e1;
                }
            }
        }
        // Block by block: while the products of block b with the state's columns and with P run, the next block's
        // residuals are corrected by the blocks before it and multiplied by its inverse.
        FragA<T, M> uf[4], f;
        float r0[4] = {}, r1[4] = {}, w0[4] = {}, w1[4] = {};
        {
            FragB<T, M> e0, e1;
            sE.b_nk(e0, e1, 0, 0);
            frag_from_acc(f, x[0], x[1]);
            mma_pair(r0, r1, w0, w1, f, e0, e1);
        }
#pragma unroll
        for (int b = 0; b < 4; ++b) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                r0[j] += w0[j], r1[j] += w1[j];
                if constexpr (kOut) x[2 * b][j] = r0[j], x[2 * b + 1][j] = r1[j];
                r0[j] *= G.beta[16 * b + 2 * t + (j & 1)];
                r1[j] *= G.beta[16 * b + 8 + 2 * t + (j & 1)];
                w0[j] = w1[j] = 0.0f;
            }
            frag_from_acc(uf[b], r0, r1);
            FragB<T, M> e0, e1;
            if (b < 3) {
#pragma unroll
                for (int j = 0; j <= b; ++j) {
                    sE.b_nk(e0, e1, b + 1, j);
                    mma_pair(x[(2 * b + 2) & 7], x[(2 * b + 3) & 7], w0, w1, uf[j], e0, e1);
                }
                sE.b_nk(e0, e1, b + 1, b + 1);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                r0[j] *= G.tail[16 * b + 2 * t + (j & 1)];
                r1[j] *= G.tail[16 * b + 8 + 2 * t + (j & 1)];
            }
            frag_from_acc(f, r0, r1);
            state_add<DK>(S, f, sK, b);
            if (b < 3) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    x[(2 * b + 2) & 7][j] += w0[j], x[(2 * b + 3) & 7][j] += w1[j];
                    r0[j] = r1[j] = w0[j] = w1[j] = 0.0f;
                }
                frag_from_acc(f, x[(2 * b + 2) & 7], x[(2 * b + 3) & 7]);
                mma_pair(r0, r1, w0, w1, f, e0, e1);
            }
            if constexpr (kOut) {
#pragma unroll
                for (int n = b; n + 1 < 4; n += 2) {
                    FragB<T, M> p[4];
                    sP.b_nk(p[0], p[1], n, b);
                    sP.b_nk(p[2], p[3], n + 1, b);
                    mma_quad(*reinterpret_cast<float(*)[4][4]>(&y[2 * n]), uf[b], p);
                }
                if ((4 - b) & 1) {
                    FragB<T, M> p0, p1;
                    float z0[4] = {}, z1[4] = {};
                    sP.b_nk(p0, p1, 3, b);
                    mma_pair(y[6], y[7], z0, z1, uf[b], p0, p1);
#pragma unroll
                    for (int j = 0; j < 4; ++j) y[6][j] += z0[j], y[7][j] += z1[j];
                }
            }
        }
        if constexpr (kOut) {
            const long long at0 = (long long)ch * kChunk * hrow;
            const int n = min(seq.len - ch * kChunk, kChunk);
            store_tokens<T>(sV, y, op + at0, hrow, n, slice * kDeltaRows, a.Dv, ovec);
            if (rp) store_tokens<T>(sV, x, rp + at0, hrow, n, slice * kDeltaRows, a.Dv, rvec);
        }
        bar_arrive(kBarEmpty + (i & 1), kChainThreads);
    }
    if constexpr (kOut) {
        if (a.final && c.segs == 1) {
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
__global__ void __launch_bounds__(kChainThreads, 1) delta_reverse_kernel(DeltaChain c) {
    using SM = ChainSmem<T, DK>;
    constexpr int M = SM::mid;
    extern __shared__ __align__(128) unsigned char smem[];
    const DeltaArgs& a = c.a;
    pdl_launch_dependents();
    pdl_wait();
    const ChainPlace at = chain_place(c, c.slices);
    const DeltaSeq seq = delta_seq(a.offsets, at.b, a.T, a.total, c.err);
    const int nc = (seq.len + kChunk - 1) / kChunk;
    const int c0 = at.seg * c.seg_chunks, c1 = min(nc, c0 + c.seg_chunks);
    if (c.segs > 1 && c0 >= nc) return;
    const long long hrow = (long long)a.Hv * a.Dv;  // do, dX and dv are dense

    if (threadIdx.x >= kStateThreads) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 128;");
        const int hk = at.h / (a.Hv / a.Hk);
        const long long brow = a.offsets ? 0 : at.b, tok0 = a.offsets ? seq.start : 0;
        const T* kp = (const T*)a.k + brow * a.k_b + tok0 * a.k_t + (long long)hk * a.Dk;
        const T* qp = (const T*)a.q + brow * a.q_b + tok0 * a.q_t + (long long)hk * a.Dk;
        const T* dp = (const T*)a.dout + seq.start * hrow + (long long)at.h * a.Dv + at.slice * kDeltaRows;
        const T* gp = (const T*)a.g + seq.start * a.Hv + at.h;
        const T* bp = (const T*)a.beta + seq.start * a.Hv + at.h;
        const int ptid = threadIdx.x - kStateThreads;
        const TileCopy<typename SM::KT, DK, kSystemThreads> ck(kp, a.k_t, a.Dk, ptid), cq(qp, a.q_t, a.Dk, ptid);
        const TileCopy<typename SM::VT, kDeltaRows, kSystemThreads> cd(dp, hrow, min(a.Dv - at.slice * kDeltaRows, kDeltaRows), ptid);
        system_warps<T, DK, true, true>(
            smem, c1 - c0, a.scale,
            [&](int i, unsigned char* s, int tid) {
                const int first = (c1 - 1 - i) * kChunk, n = min(seq.len - first, kChunk);
                ck.copy(s + SM::k, first, n, tid);
                cq.copy(s + SM::q, first, n, tid);
                cd.copy(s + SM::v, first, n, tid);
            },
            [&](int i, float(&v)[4]) {
                const int ch = c1 - 1 - i;
                const long long t0 = (long long)ch * kChunk * a.Hv;
                load_gates(gp + t0, bp + t0, min(seq.len - ch * kChunk, kChunk), a.Hv, v);
            });
        return;
    }
    asm volatile("setmaxnreg.inc.sync.aligned.u32 240;");
    const int w = threadIdx.x >> 5, t = threadIdx.x & 3, g = (threadIdx.x & 31) >> 2;
    const int row0 = at.slice * kDeltaRows + 16 * w;
    T* xp = (T*)c.dx + seq.start * hrow + (long long)at.h * a.Dv;
    T* rp = (T*)a.dv + seq.start * hrow + (long long)at.h * a.Dv;
    const bool xvec = rows_aligned(xp, hrow), rvec = rows_aligned(rp, hrow);

    float S[DK / 8][4];
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

    for (int i = 0; i < c1 - c0; ++i) {
        const int ch = c1 - 1 - i;
        unsigned char *st = smem + (i % SM::ring) * SM::stage, *sy = smem + SM::systems + (i & 1) * SM::system;
        const typename SM::KT sK(st + SM::k, kChunk), sQ(st + SM::q, kChunk);
        const typename SM::VT sD(st + SM::v, kChunk);
        const typename SM::ET sE(sy + SM::e), sP(sy + SM::p);
        const ChunkGates& G = *reinterpret_cast<const ChunkGates*>(smem + SM::gates + (i % 3) * SM::gate);
        bar_sync(kBarFull + (i & 1), kChainThreads);
        if (!c.summary)
            store_state_rows<DK>(S, (T*)c.ds + ((long long)(seq.slot + ch) * a.Hv + at.h) * a.Dv * a.Dk, row0, a.Dv, a.Dk);

        float x[8][4] = {};  // dU, then dX, transposed
        state_times<DK, false, M, T>(S, x, nullptr, sK, sK);
#pragma unroll
        for (int n = 0; n < DK / 8; ++n)
#pragma unroll
            for (int j = 0; j < 4; ++j) S[n][j] *= G.last;
#pragma unroll
        for (int n = 0; n < 8; ++n)
#pragma unroll
            for (int j = 0; j < 4; ++j) x[n][j] *= G.tail[8 * n + 2 * t + (j & 1)];
#pragma unroll
        for (int b = 0; b < 4; ++b) {  // token block b of do: P^T do into dU, (scale e^c Q)^T do into dS
            FragA<T, 1> f;
            sD.a_km(f, 16 * w, 16 * b);
#pragma unroll
            for (int n = 0; n <= b; ++n) {
                FragB<T, M> p0, p1;
                sP.b_kn(p0, p1, b, n);
                float z0[4] = {}, z1[4] = {};
                mma_pair(x[2 * n], x[2 * n + 1], z0, z1, f, p0, p1);
#pragma unroll
                for (int j = 0; j < 4; ++j) x[2 * n][j] += z0[j], x[2 * n + 1][j] += z1[j];
            }
            float d0[4], d1[4];
            sD.acc_km(d0, d1, 16 * w, 16 * b);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                d0[j] *= a.scale * G.ec[16 * b + 2 * t + (j & 1)];
                d1[j] *= a.scale * G.ec[16 * b + 8 + 2 * t + (j & 1)];
            }
            FragA<T, M> fs;
            frag_from_acc(fs, d0, d1);
            state_add<DK>(S, fs, sQ, b);
        }
        FragA<T, M> rf[4], f;
        float r0[4] = {}, r1[4] = {}, w0[4] = {}, w1[4] = {};
        {
            FragB<T, M> e0, e1;
            sE.b_kn(e0, e1, 3, 3);
            frag_from_acc(f, x[6], x[7]);
            mma_pair(r0, r1, w0, w1, f, e0, e1);
        }
#pragma unroll
        for (int b = 3; b >= 0; --b) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                r0[j] += w0[j], r1[j] += w1[j];
                x[2 * b][j] = r0[j], x[2 * b + 1][j] = r1[j];
                r0[j] *= G.beta[16 * b + 2 * t + (j & 1)];
                r1[j] *= G.beta[16 * b + 8 + 2 * t + (j & 1)];
                w0[j] = w1[j] = 0.0f;
            }
            frag_from_acc(rf[b], r0, r1);
            FragB<T, M> e0, e1;
            if (b > 0) {
#pragma unroll
                for (int j = 3; j >= b; --j) {
                    sE.b_kn(e0, e1, j, b - 1);
                    mma_pair(x[(2 * b - 2) & 7], x[(2 * b - 1) & 7], w0, w1, rf[j], e0, e1);
                }
                sE.b_kn(e0, e1, b - 1, b - 1);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                r0[j] *= -G.ec[16 * b + 2 * t + (j & 1)];
                r1[j] *= -G.ec[16 * b + 8 + 2 * t + (j & 1)];
            }
            frag_from_acc(f, r0, r1);
            state_add<DK>(S, f, sK, b);
            if (b > 0) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    x[(2 * b - 2) & 7][j] += w0[j], x[(2 * b - 1) & 7][j] += w1[j];
                    r0[j] = r1[j] = w0[j] = w1[j] = 0.0f;
                }
                frag_from_acc(f, x[(2 * b - 2) & 7], x[(2 * b - 1) & 7]);
                mma_pair(r0, r1, w0, w1, f, e0, e1);
            }
        }
        if (!c.summary) {
            const int n = min(seq.len - ch * kChunk, kChunk);
            store_tokens<T>(sD, x, xp + (long long)ch * kChunk * hrow, hrow, n, at.slice * kDeltaRows, a.Dv, xvec);
#pragma unroll
            for (int m = 0; m < 8; ++m)
#pragma unroll
                for (int j = 0; j < 4; ++j) x[m][j] *= G.beta[8 * m + 2 * t + (j & 1)];
            store_tokens<T>(sD, x, rp + (long long)ch * kChunk * hrow, hrow, n, at.slice * kDeltaRows, a.Dv, rvec);
        }
        bar_arrive(kBarEmpty + (i & 1), kChainThreads);
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
    if (!allow_smem(fn, (int)smem)) return VMB_ERR_CUDA;
    DeltaChain arg = c;
    void* args[] = {&arg};
    return launch_kernel(fn, dim3((unsigned)grid), dim3(kChainThreads), smem, args, stream) == cudaSuccess ? VMB_OK : VMB_ERR_CUDA;
}

template <typename T>
vmb_status launch_chain(const DeltaChain& c, bool reverse, cudaStream_t stream) {
    return c.a.Dk <= 64 ? launch_chain_dk<T, 64>(c, reverse, stream) : launch_chain_dk<T, 128>(c, reverse, stream);
}

}  // namespace vmb
