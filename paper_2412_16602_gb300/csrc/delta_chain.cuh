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
//
// What bounds a chain is the length of a chunk's dependent products, issued by one or two state warps per scheduler next to
// the system warps: in bf16 with Dk = 64 about 6200 cycles a chunk, 2560 of them on the tensor pipe, for 11000
// instructions of the CTA; with Dk = Dv = 128 15300, 7700 and 24100; in fp32 with Dk = 64, six tf32 products and the splits in
// place of two, 19900, 8400 and 30700.  HBM is far from it (32 images of 3136 tokens, 3 heads of 64 in bf16: 157 us, 990 GB/s).
#pragma once

#include "delta_common.cuh"
#include "delta_internal.h"
#include "vmb_internal.h"

namespace vmb {

template <typename T> struct DeltaTerms { static constexpr int mid = 2; };
template <> struct DeltaTerms<float> { static constexpr int mid = 1; };
__device__ __forceinline__ const FragA<__nv_bfloat16, 1>& lead(const FragA<__nv_bfloat16, 2>& a) {
    return reinterpret_cast<const FragA<__nv_bfloat16, 1>&>(a);
}
__device__ __forceinline__ const FragA<float, 1>& lead(const FragA<float, 1>& a) { return a; }

// Roles: the first NST warps carry the state, 16 rows each, the others load the tiles of the chunks ahead and compute
// their triangular systems.  (Done one after the other by four warps, loads and system took 8400 of a chunk's 14400 cycles
// in bf16, Dk = 64.)  Of 12 warps, four states and eight systems (240 and 128 registers a thread: 128 x 240 + 256 x 128
// is within the 384 x 168 of the launch) or, for more than 64 value channels, eight and four (256 x 208 + 128 x 88), which
// computes a system once for 128 rows.
constexpr int kChainThreads = 384;
constexpr int kBarSystem = 1, kBarFull = 2, kBarEmpty = 4;  // named barriers; full and empty: + parity of the chunk
__device__ __forceinline__ void bar_sync(int id, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }
__device__ __forceinline__ void bar_arrive(int id, int threads) { asm volatile("bar.arrive %0, %1;" ::"r"(id), "r"(threads) : "memory"); }
template <int NST> __device__ __forceinline__ void state_registers() {
    if constexpr (NST == 4)
        asm volatile("setmaxnreg.inc.sync.aligned.u32 240;");
    else
        asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
}
template <int NST> __device__ __forceinline__ void system_registers() {
    if constexpr (NST == 4)
        asm volatile("setmaxnreg.dec.sync.aligned.u32 128;");
    else
        asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
}

// Shared memory of the chain kernels, in bytes from the start: a ring of K and Q tiles, two tiles of values, two systems,
// three sets of gates.
template <typename T, int DK, int NST> struct ChainSmem {
    static constexpr int mid = DeltaTerms<T>::mid, rows = 16 * NST, states = 32 * NST, systems_n = kChainThreads - states;
    using KT = Tile<T, DK, 1>;
    using VT = Tile<T, rows, 1>;
    using ET = LowTile<T, mid>;
    static constexpr int ring = sizeof(T) == 4 && DK == 128 ? 2 : 3;
    static constexpr int k = 0, q = k + KT::bytes(kChunk), stage = q + KT::bytes(kChunk);
    static constexpr int values = ring * stage, value = VT::bytes(kChunk);
    static constexpr int e = 0, p = e + ET::kBytes, system = p + ET::kBytes;
    static constexpr int gate = (sizeof(ChunkGates) + 15) & ~15;  // a chunk's are computed ahead
    static constexpr int systems = values + 2 * value, diag = systems + 2 * system, gates = diag + 64 * 20 * 4,
                         total = gates + 3 * gate;
    static_assert(total <= 227 * 1024 && system % 16 == 0 && stage % 16 == 0 && value % 16 == 0, "fits");
};

// 16 x 64 (channel, token) accumulators of a warp to [token][channel] in global memory through the
// warp's 16 columns of a tile.
template <typename T, int ROWS>
__device__ __forceinline__ void store_tokens(const Tile<T, ROWS, 1>& s, const float (&y)[8][4], T* dst, long long stride,
                                             int rows, int ch0, int channels, bool vec) {
    const int w = threadIdx.x >> 5, lane = threadIdx.x & 31;
    constexpr int V = Tile<T, ROWS, 1>::kVec, P = 16 / V;
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

// A warp's 16 rows of the transposed state, [row][Dk] fp32 or storage type at dst (16-byte aligned).  fp32: pairs of
// columns, a sector per row and tile; bf16: the four lanes of a row exchange the pairs of four tiles, so that each
// stores the eight columns of one (1657 -> 1264 us for the training pass of 8 x 3136 tokens against single values).
template <int DK, typename T>
__device__ __forceinline__ void store_state_rows(const float (&S)[DK / 8][4], T* dst, int row0, int rows, int Dk) {
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    if (Dk % 8 == 0) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int r = row0 + g + 8 * h;
            T* p = dst + (long long)r * Dk;
            if constexpr (sizeof(T) == 2) {
#pragma unroll
                for (int q = 0; q < DK / 32; ++q) {
                    uint32_t v[4];
#pragma unroll
                    for (int n = 0; n < 4; ++n) v[n] = pack_bf16(S[4 * q + n][2 * h], S[4 * q + n][2 * h + 1]);
                    quad_transpose(v);
                    const int d = 32 * q + 8 * t;
                    if (r < rows && d < Dk) *reinterpret_cast<uint4*>(p + d) = make_uint4(v[0], v[1], v[2], v[3]);
                }
            } else {
#pragma unroll
                for (int n = 0; n < DK / 8; ++n)
                    if (r < rows && 8 * n < Dk) *reinterpret_cast<float2*>(p + 8 * n + 2 * t) = make_float2(S[n][2 * h], S[n][2 * h + 1]);
            }
        }
        return;
    }
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

// The loads and systems of the chunks of a chain, first to last or last to first, by the system warps.  `tiles` loads a
// chunk's K and Q into a stage, `values` its V or do; `gates` gives the two tokens' g and beta of a lane.
template <typename T, int DK, int NST, bool kRowBeta, bool kWithP, typename Tiles, typename Values, typename Gates>
__device__ __forceinline__ void system_warps(unsigned char* smem, int chunks, float scale, Tiles tiles, Values values, Gates gates) {
    using SM = ChainSmem<T, DK, NST>;
    constexpr int kWarps = SM::systems_n / 32, kGateWarp = kWarps - 1;
    const int tid = threadIdx.x - SM::states, w = tid >> 5;
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
        // the states are done with chunk i - 2: its system and values, and with them the oldest stage and gates, are free
        if (i >= 2) bar_sync(kBarEmpty + (i & 1), kChainThreads);
        if (!kAhead) {
            tiles(i, smem + (i % SM::ring) * SM::stage, tid);
            cp_async_commit();
        }
        values(i, smem + SM::values + (i & 1) * SM::value, tid);
        cp_async_commit();
        if (kAhead) {
            if (i + 1 < chunks) tiles(i + 1, smem + ((i + 1) % SM::ring) * SM::stage, tid);
            cp_async_commit();
            cp_async_wait<2>();  // this chunk's K and Q
        } else {
            cp_async_wait<1>();
        }
        unsigned char *st = smem + (i % SM::ring) * SM::stage, *sy = smem + SM::systems + (i & 1) * SM::system;
        bar_sync(kBarSystem, SM::systems_n);
        chunk_system<T, DK, kRowBeta, kWithP, kWarps>(typename SM::KT(st + SM::k, kChunk), typename SM::KT(st + SM::q, kChunk),
                                                      typename SM::ET(sy + SM::e), typename SM::ET(sy + SM::p), diag, gate(i), scale, w);
        if (w == kGateWarp && i + 1 < chunks) {
            chunk_gates(gate(i + 1), gv[0], gv[1], gv[2], gv[3]);
            if (i + 2 < chunks) gates(i + 2, gv);
        }
        if (kAhead) cp_async_wait<1>(); else cp_async_wait<0>();  // the values
        bar_arrive(kBarFull + (i & 1), kChainThreads);
    }
    // the last two releases, so that every barrier is left complete
    for (int i = chunks < 2 ? 0 : chunks - 2; i < chunks; ++i) bar_sync(kBarEmpty + (i & 1), kChainThreads);
}

template <typename T, typename TL> __device__ __forceinline__ void read_columns(const TL& s, int b, int d, FragB<T, 1> (&k)[4]) {
    s.b_kn(k[0], k[1], 16 * b, 32 * d);
    s.b_kn(k[2], k[3], 16 * b, 32 * d + 16);
}

// x[channel][token] += S^T K^T and, with kTwo, y += S^T Q^T (leading terms of S), the rows of the state against every
// token; the operands are read two steps (of four tiles) ahead of their products, one step where fp32
// operands, four times the registers, leave no more.
template <int DK, bool kTwo, int NS, typename T, typename TL>
__device__ __forceinline__ void state_times(const float (&S)[DK / 8][4], float (&x)[8][4], float (*y)[4], const TL& sK, const TL& sQ) {
    constexpr int kSteps = DK / 16 * (kTwo ? 4 : 2);
    constexpr int kAhead = sizeof(T) == 2 || DK == 64 ? 2 : 1;
    FragB<T, 1> b[kAhead + 1][4];
    auto read = [&](int i, FragB<T, 1>(&f)[4]) {
        const int d = kTwo ? i >> 2 : i >> 1, n = 32 * (kTwo ? (i >> 1) & 1 : i & 1);
        const TL& s = kTwo && (i & 1) ? sQ : sK;
        s.b_nk(f[0], f[1], n, 16 * d);
        s.b_nk(f[2], f[3], n + 16, 16 * d);
    };
#pragma unroll
    for (int i = 0; i < kAhead; ++i) read(i, b[i]);
    FragA<T, NS> f;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        if (i + kAhead < kSteps) read(i + kAhead, b[(i + kAhead) % (kAhead + 1)]);
        const int d = kTwo ? i >> 2 : i >> 1, n = 4 * (kTwo ? (i >> 1) & 1 : i & 1);
        if (kTwo ? i % 4 == 0 : i % 2 == 0) frag_from_acc(f, S[2 * d], S[2 * d + 1]);
        if (kTwo && (i & 1))
            mma_quad(*reinterpret_cast<float(*)[4][4]>(&y[n]), lead(f), b[i % (kAhead + 1)]);
        else
            mma_quad(*reinterpret_cast<float(*)[4][4]>(&x[n]), f, b[i % (kAhead + 1)]);
    }
}
// S += f K_b: the outer products of 16 tokens (block b of a tile) with the state's columns; `k` holds the operands of the
// first four column tiles, read before f was known.
template <int DK, int NS, typename T, typename TL>
__device__ __forceinline__ void state_add(float (&S)[DK / 8][4], const FragA<T, NS>& f, const TL& s, int b, FragB<T, 1> (&k)[2][4]) {
#pragma unroll
    for (int d = 0; d < DK / 32; ++d) {
        if (sizeof(T) == 2 || DK == 64) {
            if (d + 1 < DK / 32) read_columns(s, b, d + 1, k[(d + 1) & 1]);
        } else if (d > 0) {
            read_columns(s, b, d, k[d & 1]);
        }
        mma_quad(*reinterpret_cast<float(*)[4][4]>(&S[4 * d]), f, k[d & 1]);
    }
}

// kOut = false: the maps and sums of a segment (DeltaChain::summary).
template <typename T, int DK, int NST, bool kOut>
__global__ void __launch_bounds__(kChainThreads, 1) delta_forward_kernel(DeltaChain c) {
    using SM = ChainSmem<T, DK, NST>;
    constexpr int M = SM::mid, kRows = SM::rows;
    constexpr bool kPacked = sizeof(T) == 2;
    extern __shared__ __align__(128) unsigned char smem[];
    const DeltaArgs& a = c.a;
    pdl_launch_dependents();
    pdl_wait();
    const int vslices = c.slices, mslices = kOut ? 0 : (a.Dk + kRows - 1) / kRows;
    const ChainPlace at = chain_place(c, kOut ? vslices : (c.maps_only ? mslices : vslices + mslices));
    const bool map = !kOut && (c.maps_only || at.slice >= vslices);  // rows of the map: v = 0, S = identity
    const int slice = map && !c.maps_only ? at.slice - vslices : at.slice;
    const DeltaSeq seq = delta_seq(a.offsets, at.b, a.T, a.total, c.err);
    const int nc = chunks_of(seq.len);
    const int c0 = at.seg * c.seg_chunks, c1 = min(nc, c0 + c.seg_chunks);
    if ((!kOut || c.segs > 1) && c0 >= nc) return;
    const long long hrow = (long long)a.Hv * a.Dv;

    if (threadIdx.x >= SM::states) {
        system_registers<NST>();
        const int hk = at.h / (a.Hv / a.Hk);
        const long long brow = a.offsets ? 0 : at.b, tok0 = a.offsets ? seq.start : 0;
        const T* kp = (const T*)a.k + brow * a.k_b + tok0 * a.k_t + (long long)hk * a.Dk;
        const T* qp = (const T*)a.q + brow * a.q_b + tok0 * a.q_t + (long long)hk * a.Dk;
        const T* vp = (const T*)a.v + brow * a.v_b + tok0 * a.v_t + (long long)at.h * a.Dv + slice * kRows;
        const T* gp = (const T*)a.g + seq.start * a.Hv + at.h;
        const T* bp = (const T*)a.beta + seq.start * a.Hv + at.h;
        const int ptid = threadIdx.x - SM::states;
        const TileCopy<typename SM::KT, DK, SM::systems_n> ck(kp, a.k_t, a.Dk, ptid), cq(qp, a.q_t, a.Dk, ptid);
        const TileCopy<typename SM::VT, kRows, SM::systems_n> cv(vp, a.v_t, min(a.Dv - slice * kRows, kRows), ptid);
        system_warps<T, DK, NST, false, kOut>(
            smem, c1 - c0, a.scale,
            [&](int i, unsigned char* s, int tid) {
                const int first = (c0 + i) * kChunk, n = min(seq.len - first, kChunk);
                ck.copy(s + SM::k, first, n, tid);
                if (kOut) cq.copy(s + SM::q, first, n, tid);
            },
            [&](int i, unsigned char* s, int tid) {
                const int first = (c0 + i) * kChunk;
                if (!map) cv.copy(s, first, min(seq.len - first, kChunk), tid);
            },
            [&](int i, float(&v)[4]) {
                const long long t0 = (long long)(c0 + i) * kChunk * a.Hv;
                load_gates(gp + t0, bp + t0, min(seq.len - (c0 + i) * kChunk, kChunk), a.Hv, v);
            });
        return;
    }
    state_registers<NST>();
    const int w = threadIdx.x >> 5, t = threadIdx.x & 3, g = (threadIdx.x & 31) >> 2;
    const int row0 = slice * kRows + 16 * w;
    T* op = kOut ? (T*)a.o + seq.start * hrow + (long long)at.h * a.Dv : nullptr;
    T* rp = kOut && a.saved_r ? (T*)a.saved_r + seq.start * hrow + (long long)at.h * a.Dv : nullptr;
    const bool ovec = kOut && rows_aligned(op, hrow), rvec = kOut && rows_aligned(rp, hrow);

    float S[DK / 8][4];
    if (kOut && c.segs > 1) {
        load_state_rows<DK>(S, c.sums + (at.chain * c.segs + at.seg) * a.Dv * DK, row0, a.Dv, DK, DK, 1);
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
        const typename SM::VT sV(smem + SM::values + (i & 1) * SM::value, kChunk);
        const typename SM::ET sE(sy + SM::e), sP(sy + SM::p);
        const ChunkGates& G = *reinterpret_cast<const ChunkGates*>(smem + SM::gates + (i % 3) * SM::gate);
        bar_sync(kBarFull + (i & 1), kChainThreads);
        if (kOut && a.saved)
            store_state_rows<DK>(S, (T*)a.saved + ((long long)(seq.slot + ch) * a.Hv + at.h) * a.Dv * a.Dk, row0, a.Dv, a.Dk);

        float x[8][4] = {}, y[kOut ? 8 : 1][4] = {};  // K S and Q S, transposed: [channel][token]
        state_times<DK, kOut, M, T>(S, x, y, sK, sQ);
#pragma unroll
        for (int n = 0; n < DK / 8; ++n) scale4<kPacked>(S[n], make_float2(G.last, G.last));
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            float v0[4] = {}, v1[4] = {};
            if (!map) sV.acc_km(v0, v1, 16 * w, 16 * n);
            const float2 e0 = G.pair(G.ec, 2 * n), e1 = G.pair(G.ec, 2 * n + 1);
            if constexpr (kOut) {
                scale4<kPacked>(y[2 * n], make_float2(a.scale * e0.x, a.scale * e0.y));
                scale4<kPacked>(y[2 * n + 1], make_float2(a.scale * e1.x, a.scale * e1.y));
            }
            const float2 m0 = make_float2(-e0.x, -e0.y), m1 = make_float2(-e1.x, -e1.y);
            if constexpr (kPacked) {
                put4(x[2 * n], __ffma2_rn(lo2(x[2 * n]), m0, lo2(v0)), __ffma2_rn(hi2(x[2 * n]), m0, hi2(v0)));
                put4(x[2 * n + 1], __ffma2_rn(lo2(x[2 * n + 1]), m1, lo2(v1)), __ffma2_rn(hi2(x[2 * n + 1]), m1, hi2(v1)));
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    x[2 * n][j] = fmaf(x[2 * n][j], j & 1 ? m0.y : m0.x, v0[j]);
                    x[2 * n + 1][j] = fmaf(x[2 * n + 1][j], j & 1 ? m1.y : m1.x, v1[j]);
                }
            }
        }
        // Block by block: while the products of block b with the state's columns and with P run, the next block's
        // residuals are corrected by the blocks before it and multiplied by its inverse.  Operands that do not depend
        // on the residuals are read ahead.
        FragA<T, M> uf[4], f;
        constexpr bool kEarly = sizeof(T) == 2 || DK == 64;
        FragB<T, M> e[4][2];
        FragB<T, 1> kc[2][4];
        float r0[4] = {}, r1[4] = {}, w0[4] = {}, w1[4] = {};
        sE.b_nk(e[0][0], e[0][1], 0, 0);
        frag_from_acc(f, x[0], x[1]);
        mma_pair(r0, r1, w0, w1, f, e[0][0], e[0][1]);
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            if (kEarly) read_columns(sK, b, 0, kc[0]);
            if (kEarly && b < 3) {
#pragma unroll
                for (int j = 0; j <= b + 1; ++j) sE.b_nk(e[j][0], e[j][1], b + 1, j);
            }
            const float2 b0 = G.pair(G.beta, 2 * b), b1 = G.pair(G.beta, 2 * b + 1), t0 = G.pair(G.tail, 2 * b), t1 = G.pair(G.tail, 2 * b + 1);
            add4<kPacked>(r0, w0), add4<kPacked>(r1, w1);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (kOut) x[2 * b][j] = r0[j], x[2 * b + 1][j] = r1[j];
                w0[j] = w1[j] = 0.0f;
            }
            scale4<kPacked>(r0, b0), scale4<kPacked>(r1, b1);
            frag_from_acc(uf[b], r0, r1);
            if (b < 3) {
#pragma unroll
                for (int j = 0; j <= b; ++j) {
                    if (!kEarly) sE.b_nk(e[j][0], e[j][1], b + 1, j);
                    mma_pair(x[(2 * b + 2) & 7], x[(2 * b + 3) & 7], w0, w1, uf[j], e[j][0], e[j][1]);
                }
            }
            scale4<kPacked>(r0, t0), scale4<kPacked>(r1, t1);
            frag_from_acc(f, r0, r1);
            if (!kEarly) read_columns(sK, b, 0, kc[0]);
            state_add<DK>(S, f, sK, b, kc);
            FragB<T, M> p[4];
            if constexpr (kOut) {
                if (b < 3) {
                    sP.b_nk(p[0], p[1], b, b);
                    sP.b_nk(p[2], p[3], b + 1, b);
                }
            }
            if (b < 3) {
                add4<kPacked>(x[(2 * b + 2) & 7], w0), add4<kPacked>(x[(2 * b + 3) & 7], w1);
#pragma unroll
                for (int j = 0; j < 4; ++j) r0[j] = r1[j] = w0[j] = w1[j] = 0.0f;
                frag_from_acc(f, x[(2 * b + 2) & 7], x[(2 * b + 3) & 7]);
                if (!kEarly) sE.b_nk(e[(b + 1) & 3][0], e[(b + 1) & 3][1], b + 1, b + 1);
                mma_pair(r0, r1, w0, w1, f, e[(b + 1) & 3][0], e[(b + 1) & 3][1]);
            }
            if constexpr (kOut) {
                if (b < 3) mma_quad(*reinterpret_cast<float(*)[4][4]>(&y[2 * b]), uf[b], p);
                if (b == 0) {
                    sP.b_nk(p[0], p[1], 2, 0);
                    sP.b_nk(p[2], p[3], 3, 0);
                    mma_quad(*reinterpret_cast<float(*)[4][4]>(&y[4]), uf[0], p);
                }
                if (b == 1 || b == 3) {
                    float z0[4] = {}, z1[4] = {};
                    sP.b_nk(p[0], p[1], 3, b);
                    mma_pair(y[6], y[7], z0, z1, uf[b], p[0], p[1]);
                    add4<kPacked>(y[6], z0), add4<kPacked>(y[7], z1);
                }
            }
        }
        if constexpr (kOut) {
            const long long at0 = (long long)ch * kChunk * hrow;
            const int n = min(seq.len - ch * kChunk, kChunk);
            store_tokens<T, kRows>(sV, y, op + at0, hrow, n, slice * kRows, a.Dv, ovec);
            if (rp) store_tokens<T, kRows>(sV, x, rp + at0, hrow, n, slice * kRows, a.Dv, rvec);
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
        if (map && c.maps_only) {  // for the reverse: transposed
#pragma unroll
            for (int n = 0; n < DK / 8; ++n)
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const int r = row0 + g + 8 * (x >> 1), d = 8 * n + 2 * t + (x & 1);
                    if (r < DK) c.maps[(i * DK + d) * DK + r] = S[n][x];
                }
        } else if (map) {
            store_state_rows<DK>(S, c.maps + i * DK * DK, row0, DK, DK);
        } else {
            store_state_rows<DK>(S, c.sums + i * a.Dv * DK, row0, a.Dv, DK);
        }
    }
}

// The reverse: dS (transposed, like S) from the last chunk to the first,
//   dU = P^T do + tail K dS,  dX = (I + b E)^-T dU,  dR = b dX,
//   dS <- e^(c_last) dS + (scale e^c Q)^T do - (e^c K)^T dR.
// Writes dS at each chunk's end, dX and dv = dR of every token; with DeltaChain::summary only the segment's sum.
template <typename T, int DK, int NST>
__global__ void __launch_bounds__(kChainThreads, 1) delta_reverse_kernel(DeltaChain c) {
    using SM = ChainSmem<T, DK, NST>;
    constexpr int M = SM::mid, kRows = SM::rows;
    constexpr bool kPacked = sizeof(T) == 2;
    extern __shared__ __align__(128) unsigned char smem[];
    const DeltaArgs& a = c.a;
    pdl_launch_dependents();
    pdl_wait();
    const ChainPlace at = chain_place(c, c.slices);
    const DeltaSeq seq = delta_seq(a.offsets, at.b, a.T, a.total, c.err);
    const int nc = chunks_of(seq.len);
    const int c0 = at.seg * c.seg_chunks, c1 = min(nc, c0 + c.seg_chunks);
    if (c.segs > 1 && c0 >= nc) return;
    const long long hrow = (long long)a.Hv * a.Dv;  // do, dX and dv are dense

    if (threadIdx.x >= SM::states) {
        system_registers<NST>();
        const int hk = at.h / (a.Hv / a.Hk);
        const long long brow = a.offsets ? 0 : at.b, tok0 = a.offsets ? seq.start : 0;
        const T* kp = (const T*)a.k + brow * a.k_b + tok0 * a.k_t + (long long)hk * a.Dk;
        const T* qp = (const T*)a.q + brow * a.q_b + tok0 * a.q_t + (long long)hk * a.Dk;
        const T* dp = (const T*)a.dout + seq.start * hrow + (long long)at.h * a.Dv + at.slice * kRows;
        const T* gp = (const T*)a.g + seq.start * a.Hv + at.h;
        const T* bp = (const T*)a.beta + seq.start * a.Hv + at.h;
        const int ptid = threadIdx.x - SM::states;
        const TileCopy<typename SM::KT, DK, SM::systems_n> ck(kp, a.k_t, a.Dk, ptid), cq(qp, a.q_t, a.Dk, ptid);
        const TileCopy<typename SM::VT, kRows, SM::systems_n> cd(dp, hrow, min(a.Dv - at.slice * kRows, kRows), ptid);
        system_warps<T, DK, NST, true, true>(
            smem, c1 - c0, a.scale,
            [&](int i, unsigned char* s, int tid) {
                const int first = (c1 - 1 - i) * kChunk, n = min(seq.len - first, kChunk);
                ck.copy(s + SM::k, first, n, tid);
                cq.copy(s + SM::q, first, n, tid);
            },
            [&](int i, unsigned char* s, int tid) {
                const int first = (c1 - 1 - i) * kChunk;
                cd.copy(s, first, min(seq.len - first, kChunk), tid);
            },
            [&](int i, float(&v)[4]) {
                const int ch = c1 - 1 - i;
                const long long t0 = (long long)ch * kChunk * a.Hv;
                load_gates(gp + t0, bp + t0, min(seq.len - ch * kChunk, kChunk), a.Hv, v);
            });
        return;
    }
    state_registers<NST>();
    const int w = threadIdx.x >> 5, t = threadIdx.x & 3, g = (threadIdx.x & 31) >> 2;
    const int row0 = at.slice * kRows + 16 * w;
    T* xp = (T*)c.dx + seq.start * hrow + (long long)at.h * a.Dv;
    T* rp = (T*)a.dv + seq.start * hrow + (long long)at.h * a.Dv;
    const bool xvec = rows_aligned(xp, hrow), rvec = rows_aligned(rp, hrow);

    float S[DK / 8][4];
    if (!c.summary && c.segs > 1) {
        load_state_rows<DK>(S, c.sums + (at.chain * c.segs + at.seg) * a.Dv * DK, row0, a.Dv, DK, DK, 1);
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
        const typename SM::VT sD(smem + SM::values + (i & 1) * SM::value, kChunk);
        const typename SM::ET sE(sy + SM::e), sP(sy + SM::p);
        const ChunkGates& G = *reinterpret_cast<const ChunkGates*>(smem + SM::gates + (i % 3) * SM::gate);
        bar_sync(kBarFull + (i & 1), kChainThreads);
        if (!c.summary)
            store_state_rows<DK>(S, (T*)c.ds + ((long long)(seq.slot + ch) * a.Hv + at.h) * a.Dv * a.Dk, row0, a.Dv, a.Dk);

        float x[8][4] = {};  // dU, then dX, transposed
        state_times<DK, false, M, T>(S, x, nullptr, sK, sK);
#pragma unroll
        for (int n = 0; n < DK / 8; ++n) scale4<kPacked>(S[n], make_float2(G.last, G.last));
#pragma unroll
        for (int n = 0; n < 8; ++n) scale4<kPacked>(x[n], G.pair(G.tail, n));
        FragB<T, 1> kc[2][4];
#pragma unroll
        for (int b = 0; b < 4; ++b) {  // token block b of do: P^T do into dU, (scale e^c Q)^T do into dS
            FragA<T, 1> f;
            sD.a_km(f, 16 * w, 16 * b);
            read_columns(sQ, b, 0, kc[0]);
            float d0[4], d1[4];
            sD.acc_km(d0, d1, 16 * w, 16 * b);
            const float2 e0 = G.pair(G.ec, 2 * b), e1 = G.pair(G.ec, 2 * b + 1);
            scale4<kPacked>(d0, make_float2(a.scale * e0.x, a.scale * e0.y));
            scale4<kPacked>(d1, make_float2(a.scale * e1.x, a.scale * e1.y));
            FragA<T, M> fs;
            frag_from_acc(fs, d0, d1);
#pragma unroll
            for (int n = 0; n + 1 <= b; n += 2) {
                FragB<T, M> p[4];
                sP.b_kn(p[0], p[1], b, n);
                sP.b_kn(p[2], p[3], b, n + 1);
                mma_quad(*reinterpret_cast<float(*)[4][4]>(&x[2 * n]), f, p);
            }
            if (b % 2 == 0) {
                FragB<T, M> p0, p1;
                sP.b_kn(p0, p1, b, b);
                float z0[4] = {}, z1[4] = {};
                mma_pair(x[2 * b], x[2 * b + 1], z0, z1, f, p0, p1);
                add4<kPacked>(x[2 * b], z0), add4<kPacked>(x[2 * b + 1], z1);
            }
            state_add<DK>(S, fs, sQ, b, kc);
        }
        constexpr bool kEarly = sizeof(T) == 2 || DK == 64;
        FragA<T, M> rf[4], f;
        FragB<T, M> e[4][2];
        float r0[4] = {}, r1[4] = {}, w0[4] = {}, w1[4] = {};
        sE.b_kn(e[3][0], e[3][1], 3, 3);
        frag_from_acc(f, x[6], x[7]);
        mma_pair(r0, r1, w0, w1, f, e[3][0], e[3][1]);
#pragma unroll
        for (int b = 3; b >= 0; --b) {
            if (kEarly) read_columns(sK, b, 0, kc[0]);
            if (kEarly && b > 0) {
#pragma unroll
                for (int j = 3; j >= b - 1; --j) sE.b_kn(e[j][0], e[j][1], j, b - 1);
            }
            const float2 b0 = G.pair(G.beta, 2 * b), b1 = G.pair(G.beta, 2 * b + 1), t0 = G.pair(G.ec, 2 * b), t1 = G.pair(G.ec, 2 * b + 1);
            add4<kPacked>(r0, w0), add4<kPacked>(r1, w1);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                x[2 * b][j] = r0[j], x[2 * b + 1][j] = r1[j];
                w0[j] = w1[j] = 0.0f;
            }
            scale4<kPacked>(r0, b0), scale4<kPacked>(r1, b1);
            frag_from_acc(rf[b], r0, r1);
            if (b > 0) {
#pragma unroll
                for (int j = 3; j >= b; --j) {
                    if (!kEarly) sE.b_kn(e[j][0], e[j][1], j, b - 1);
                    mma_pair(x[(2 * b - 2) & 7], x[(2 * b - 1) & 7], w0, w1, rf[j], e[j][0], e[j][1]);
                }
            }
            scale4<kPacked>(r0, make_float2(-t0.x, -t0.y)), scale4<kPacked>(r1, make_float2(-t1.x, -t1.y));
            frag_from_acc(f, r0, r1);
            if (!kEarly) read_columns(sK, b, 0, kc[0]);
            state_add<DK>(S, f, sK, b, kc);
            if (b > 0) {
                add4<kPacked>(x[(2 * b - 2) & 7], w0), add4<kPacked>(x[(2 * b - 1) & 7], w1);
#pragma unroll
                for (int j = 0; j < 4; ++j) r0[j] = r1[j] = w0[j] = w1[j] = 0.0f;
                frag_from_acc(f, x[(2 * b - 2) & 7], x[(2 * b - 1) & 7]);
                if (!kEarly) sE.b_kn(e[(b - 1) & 3][0], e[(b - 1) & 3][1], b - 1, b - 1);
                mma_pair(r0, r1, w0, w1, f, e[(b - 1) & 3][0], e[(b - 1) & 3][1]);
            }
        }
        if (!c.summary) {
            const int n = min(seq.len - ch * kChunk, kChunk);
            store_tokens<T, kRows>(sD, x, xp + (long long)ch * kChunk * hrow, hrow, n, at.slice * kRows, a.Dv, xvec);
#pragma unroll
            for (int m = 0; m < 8; ++m) scale4<kPacked>(x[m], G.pair(G.beta, m));
            store_tokens<T, kRows>(sD, x, rp + (long long)ch * kChunk * hrow, hrow, n, at.slice * kRows, a.Dv, rvec);
        }
        bar_arrive(kBarEmpty + (i & 1), kChainThreads);
    }
    if (c.summary) {
        store_state_rows<DK>(S, c.sums + (at.chain * c.segs + at.seg) * a.Dv * DK, row0, a.Dv, DK);
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

template <typename T, int DK, int NST>
vmb_status launch_chain_dk(const DeltaChain& c, bool reverse, cudaStream_t stream) {
    const void* fn = reverse ? (const void*)delta_reverse_kernel<T, DK, NST>
                             : c.summary ? (const void*)delta_forward_kernel<T, DK, NST, false> : (const void*)delta_forward_kernel<T, DK, NST, true>;
    DeltaChain arg = c;
    arg.slices = (c.a.Dv + 16 * NST - 1) / (16 * NST);
    const int mslices = (c.a.Dk + 16 * NST - 1) / (16 * NST);
    const long long per = reverse || !c.summary ? arg.slices : c.maps_only ? mslices : arg.slices + mslices;
    const long long grid = (long long)c.a.B * c.a.Hv * c.segs * per;
    const size_t smem = ChainSmem<T, DK, NST>::total;
    if (!allow_smem(fn, (int)smem)) return VMB_ERR_CUDA;
    void* args[] = {&arg};
    // A grid of less than one wave is launched when the previous kernel has completed: its CTAs live long, and launched
    // early they wait on the SMs that become free first (the three launches of one 3136-token image took 167 us instead of
    // 97, with three chunks a segment and a slower walk; 96 chains 185 us instead of 165).
    return launch_kernel(fn, dim3((unsigned)grid), dim3(kChainThreads), smem, args, stream, grid > device_sm_count()) == cudaSuccess
               ? VMB_OK : VMB_ERR_CUDA;
}

template <typename T>
vmb_status launch_chain(const DeltaChain& c, bool reverse, cudaStream_t stream) {
    if constexpr (sizeof(T) == 2)
        if (c.wide) return c.a.Dk <= 64 ? launch_chain_dk<T, 64, 8>(c, reverse, stream) : launch_chain_dk<T, 128, 8>(c, reverse, stream);
    return c.a.Dk <= 64 ? launch_chain_dk<T, 64, 4>(c, reverse, stream) : launch_chain_dk<T, 128, 4>(c, reverse, stream);
}

}  // namespace vmb
