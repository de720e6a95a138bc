// delta_grad.cuh - the gradients of the gated delta rule that are local to a chunk, once the state S
// before it, the gradient dS of the state after it, the residuals r and dX are known (u = b r, dR = b dX):
//   dP_ij = scale e^(c_i - c_j) do_i.u_j (j <= i),   dA_ij = -e^(c_i - c_j) dR_i.u_j (j < i),
//   dq = scale e^c do S^T + dP k,
//   dk = -e^c dR S^T + tail u dS^T + dA k + dA^T k + dP^T q,   dbeta_i = dX_i.r_i,
//   dc: row sums minus column sums of dP.(q k^T) + dA.(k k^T), q.dq and k.dk of the products with S,
//       minus k.dk of the product with dS; all of the latter and e^(c_last) <S, dS> at the last token;
//   dg_t = sum of dc_i over i >= t of the chunk.
// (The pairs within i, j >= t cancel in dg: taken from the same fp32 products they do so exactly up to
// fp32 rounding, which q.dq - k.dk of the finished gradients, rounded through bf16 operands, would not.)
//
// One CTA per chunk and key head takes the value heads that share it in turn and sums their dq and dk in shared
// memory (fp32 with Dk > 64 has no room for the sums: one CTA per value head, the sums by delta_share_kernel).  Warp w
// computes the 16 tokens of block w % 4 for a part of the Dk columns, and a part of the 64 x 64 products dP or dA.  The
// value channels come in slices of 64, the next slice on its way while one is multiplied where it fits.  Scales by
// token are applied to the accumulators, so that the operands are the kept values themselves.
// The kept states and residuals and the dS and dX of the reverse pass have the storage type.  For bf16 they are most of what a
// training pass moves, and their rounding reaches one chunk's gradients, never the state: dg and dbeta, sums of many of their
// products, are off by 0.0029 of their size (rms) where rounding the results alone gives 0.0017; dq, dk and dv by that alone.
//
// Bound by latency within a chunk: at four warps per scheduler an instruction issues in 40 to 47% of the cycles, the tensor
// pipe works in 25 to 31% of them, DRAM at 13 to 19% (8 x 3136 tokens of 12 heads of 128 x 128 over 6 key heads in bf16: 457 us;
// 32 x 784 tokens of 6 heads of 64 x 64 in fp32: 329 us, cold and on its own).
#pragma once

#include "delta_common.cuh"
#include "delta_internal.h"

namespace vmb {

// bf16 with Dk <= 64: eight warps and two CTAs per SM, whose loads and products overlap; otherwise 16 warps, or eight
// of 255 registers where 128 are too few (fp32 with Dk > 64: 1.2 KB of spills per thread).
template <typename T, int DK> struct GradSmem {
    static constexpr bool small = sizeof(T) == 2 && DK == 64;
    static constexpr int warps = small || (sizeof(T) == 4 && DK == 128) ? 8 : 16, threads = 32 * warps, groups = warps / 4;
    using KT = Tile<T, DK, 1>;
    using VT = Tile<T, 64, 1>;
    using PT = Tile<T, 64, sizeof(T) == 2 ? 2 : 1>;
    // a slice: do, r, dX, S, dS; dP and dA take the place of the last one read
    static constexpr int d = 0, r = d + VT::bytes(64), x = r + VT::bytes(64), s = x + VT::bytes(64), ds = s + KT::bytes(64),
                         slice = ds + KT::bytes(64);
    static constexpr int dp = 0, da = dp + PT::bytes(64);
    static_assert(da + PT::bytes(64) <= slice, "dP and dA fit");
    // row sums [groups][64], column sums [2][4][64], dots [groups][3][64], dbeta [64], block sums [16]
    static constexpr int sums = (groups * 64 + 512 + groups * 192 + 64 + 16) * 4;
    static constexpr int k = 0, q = k + KT::bytes(64), gates = q + KT::bytes(64),
                         sum0 = gates + (((int)sizeof(ChunkGates) + 15) & ~15), slices = (sum0 + sums + 127) & ~127;
    static constexpr int limit = small ? 113 * 1024 : 227 * 1024;
    static constexpr bool totals = slices + slice + 2 * 64 * DK * 4 <= limit;
    static constexpr int tot = slices + slice, one = tot + (totals ? 2 * 64 * DK * 4 : 0);
    static constexpr bool ahead = !small && one + slice <= limit;  // a second slice
    static constexpr int slice2 = one, total = one + (ahead ? slice : 0);
    static_assert(total <= limit, "fits");
};

template <typename T, int DK>
__global__ void __launch_bounds__(GradSmem<T, DK>::threads, GradSmem<T, DK>::small ? 2 : 1) delta_grad_kernel(DeltaGrad c) {
    using SM = GradSmem<T, DK>;
    constexpr int N = SM::threads, NG = SM::groups, HC = DK / NG, HT = HC / 8;  // columns and column tiles per warp
    constexpr int JB = 8 / NG;                                                   // blocks of dP or dA per warp
    extern __shared__ __align__(128) unsigned char smem[];
    const DeltaArgs& a = c.a;
    const int tid = threadIdx.x, w = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    const int tb = w & 3, qt = w >> 2, col0 = qt * HC;
    const bool second = qt & 1;  // this warp's part of dA, otherwise of dP
    auto block = [&](int i) { return NG == 2 ? i : 2 * i + (qt >> 1); };
    pdl_launch_dependents();
    pdl_wait();
    const int chunks = chunks_of(a.T), share = a.Hv / a.Hk, heads = SM::totals ? a.Hk : a.Hv;
    const int ch = blockIdx.x % chunks;
    const long long chain = blockIdx.x / chunks;
    const int head = (int)(chain % heads), b = (int)(chain / heads);
    const DeltaSeq seq = delta_seq(a.offsets, b, a.T, a.total, c.err);
    const int n = min(seq.len - ch * kChunk, kChunk);
    if (n <= 0) return;
    const int hk = SM::totals ? head : head / share, h0 = SM::totals ? head * share : head, turns = SM::totals ? share : 1;
    const long long brow = a.offsets ? 0 : b, tok0 = (a.offsets ? seq.start : 0) + (long long)ch * kChunk;
    const long long tok = seq.start + (long long)ch * kChunk;  // in the dense tensors
    const T* kp = (const T*)a.k + brow * a.k_b + tok0 * a.k_t + (long long)hk * a.Dk;
    const T* qp = (const T*)a.q + brow * a.q_b + tok0 * a.q_t + (long long)hk * a.Dk;
    const long long hrow = (long long)a.Hv * a.Dv;

    const typename SM::KT sK(smem + SM::k, 64), sQ(smem + SM::q, 64);
    ChunkGates& G = *reinterpret_cast<ChunkGates*>(smem + SM::gates);
    float* rowsum = reinterpret_cast<float*>(smem + SM::sum0);
    float *colsum = rowsum + NG * 64, *dots = colsum + 512, *dbeta = dots + NG * 192, *blocks = dbeta + 64;
    float* tot = reinterpret_cast<float*>(smem + SM::tot);
    const int vslices = (a.Dv + 63) / 64, steps = turns * vslices;

    // slice i of the CTA: value head h0 + i / vslices, channels from 64 (i % vslices)
    auto load = [&](int i) {
        const int h = h0 + i / vslices, v0 = (i % vslices) * 64, cols = min(a.Dv - v0, 64);
        unsigned char* s = smem + (SM::ahead && (i & 1) ? SM::slice2 : SM::slices);
        const long long off = tok * hrow + (long long)h * a.Dv + v0;
        const T *dp = (const T*)a.dout + off, *rp = (const T*)a.saved_r + off, *xp = (const T*)c.dx + off;
        load_tile<64, 64>(typename SM::VT(s + SM::d, 64), dp, hrow, n, cols, rows_aligned(dp, hrow), tid, N);
        load_tile<64, 64>(typename SM::VT(s + SM::r, 64), rp, hrow, n, cols, rows_aligned(rp, hrow), tid, N);
        load_tile<64, 64>(typename SM::VT(s + SM::x, 64), xp, hrow, n, cols, rows_aligned(xp, hrow), tid, N);
        const long long srow = (((long long)(seq.slot + ch) * a.Hv + h) * a.Dv + v0) * a.Dk;
        const T *sp = (const T*)a.saved + srow, *dsp = (const T*)c.ds + srow;
        load_tile<64, DK>(typename SM::KT(s + SM::s, 64), sp, a.Dk, cols, a.Dk, rows_aligned(sp, a.Dk), tid, N);
        load_tile<64, DK>(typename SM::KT(s + SM::ds, 64), dsp, a.Dk, cols, a.Dk, rows_aligned(dsp, a.Dk), tid, N);
        cp_async_commit();
    };
    load_tile<64, DK>(sK, kp, a.k_t, n, a.Dk, rows_aligned(kp, a.k_t), tid, N);
    load_tile<64, DK>(sQ, qp, a.q_t, n, a.Dk, rows_aligned(qp, a.q_t), tid, N);
    load(0);

    float dq[HT][4], dkr[HT][4], dkt[HT][4], W[2 * JB][4];
    float2 sdot = make_float2(0.0f, 0.0f), bdot = sdot;
    for (int i = 0; i < steps; ++i) {
        const int h = h0 + i / vslices, vs = i % vslices;
        unsigned char* s = smem + (SM::ahead && (i & 1) ? SM::slice2 : SM::slices);
        const typename SM::KT sS(s + SM::s, 64), sDS(s + SM::ds, 64);
        const typename SM::VT sD(s + SM::d, 64), sR(s + SM::r, 64), sX(s + SM::x, 64);
        if (vs == 0) {
#pragma unroll
            for (int j = 0; j < HT; ++j)
#pragma unroll
                for (int x = 0; x < 4; ++x) dq[j][x] = dkr[j][x] = dkt[j][x] = 0.0f;
#pragma unroll
            for (int j = 0; j < 2 * JB; ++j)
#pragma unroll
                for (int x = 0; x < 4; ++x) W[j][x] = 0.0f;
            sdot = bdot = make_float2(0.0f, 0.0f);
            if (w == 0) {
                const T *gp = (const T*)a.g + tok * a.Hv + h, *bp = (const T*)a.beta + tok * a.Hv + h;
                float v[4];
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    v[x] = 2 * lane + x < n ? io<T>::cvt(gp[(long long)(2 * lane + x) * a.Hv]) : 0.0f;
                    v[2 + x] = 2 * lane + x < n ? io<T>::cvt(bp[(long long)(2 * lane + x) * a.Hv]) : 0.0f;
                }
                chunk_gates(G, v[0], v[1], v[2], v[3]);
            }
        }
        if (SM::ahead && i + 1 < steps) {
            load(i + 1);
            cp_async_wait<1>();
        } else {
            cp_async_wait<0>();
        }
        __syncthreads();
        {  // this thread's part of dbeta: token tid / (N / 64); and of <S, dS>
            constexpr int per = N / 64, Vv = SM::KT::kVec;
            const int tk = tid / per, p = tid % per;
#pragma unroll
            for (int j = 0; j < 64 / (per * Vv); ++j) sX.dot_vec(sR, tk, (p + per * j) * Vv, bdot);
#pragma unroll 2
            for (int j = tid; j < 64 * DK / Vv; j += N) sS.dot_vec(sDS, j / (DK / Vv), j % (DK / Vv) * Vv, sdot);
        }
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
            FragA<T, 1> fd, fx, fr;
            sD.a_mk(fd, 16 * tb, 16 * kk);
            sX.a_mk(fx, 16 * tb, 16 * kk);
            sR.a_mk(fr, 16 * tb, 16 * kk);
            FragB<T, 1> b0, b1;
#pragma unroll
            for (int j = 0; j < HT / 2; ++j) {
                sS.b_kn(b0, b1, 16 * kk, col0 + 16 * j);
                mma16(dq[2 * j], fd, b0);
                mma16(dq[2 * j + 1], fd, b1);
                mma16(dkr[2 * j], fx, b0);
                mma16(dkr[2 * j + 1], fx, b1);
                sDS.b_kn(b0, b1, 16 * kk, col0 + 16 * j);
                mma16(dkt[2 * j], fr, b0);
                mma16(dkt[2 * j + 1], fr, b1);
            }
#pragma unroll
            for (int j = 0; j < JB; ++j)
                if (block(j) <= tb) {
                    sR.b_nk(b0, b1, 16 * block(j), 16 * kk);
                    mma16(W[2 * j], second ? fx : fd, b0);
                    mma16(W[2 * j + 1], second ? fx : fd, b1);
                }
        }
        if (vs + 1 < vslices) {
            __syncthreads();  // this slice has been read
            if (!SM::ahead) load(i + 1);
            continue;
        }
        // dP or dA, and their products with q k^T or k k^T
        const typename SM::PT sDP(s + SM::dp, 64), sDA(s + SM::da, 64);
        float rs[2] = {};
        {
            float m[2 * JB][4] = {};
#pragma unroll
            for (int d = 0; d < DK / 16; ++d) {
                FragA<T, 1> f;
                FragB<T, 1> b0, b1;
                if (second) sK.a_mk(f, 16 * tb, 16 * d); else sQ.a_mk(f, 16 * tb, 16 * d);
#pragma unroll
                for (int j = 0; j < JB; ++j)
                    if (block(j) <= tb) {
                        sK.b_nk(b0, b1, 16 * block(j), 16 * d);
                        mma16(m[2 * j], f, b0);
                        mma16(m[2 * j + 1], f, b1);
                    }
            }
            __syncthreads();  // do, r, dX, S and dS have been read
#pragma unroll
            for (int jt = 0; jt < 2 * JB; ++jt) {
                const int bj = block(jt / 2), j0 = 16 * bj + 8 * (jt & 1) + 2 * t;
                float cs[2] = {};
                if (bj <= tb) {
                    const float2 jh = *reinterpret_cast<const float2*>(G.hi + j0), jl = *reinterpret_cast<const float2*>(G.lo + j0),
                                 jb = *reinterpret_cast<const float2*>(G.beta + j0);
#pragma unroll
                    for (int hh = 0; hh < 2; ++hh) {
                        const int r = 16 * tb + g + 8 * hh;
                        const float ih = G.hi[r], il = G.lo[r], sc = second ? -G.beta[r] : a.scale;
                        const float e0 = ex2((ih - jh.x) + (il - jl.x)) * (sc * jb.x), e1 = ex2((ih - jh.y) + (il - jl.y)) * (sc * jb.y);
                        // (above the diagonal the exponential may be anything: not taken)
                        const float v[2] = {j0 + second <= r ? e0 * W[jt][2 * hh] : 0.0f, j0 + 1 + second <= r ? e1 * W[jt][2 * hh + 1] : 0.0f};
                        const float p0 = v[0] * m[jt][2 * hh], p1 = v[1] * m[jt][2 * hh + 1];
                        rs[hh] += p0 + p1;
                        cs[0] += p0;
                        cs[1] += p1;
                        (second ? sDA : sDP).set2(r, j0, v[0], v[1]);
                    }
                }
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    cs[x] += __shfl_xor_sync(0xffffffffu, cs[x], 4);
                    cs[x] += __shfl_xor_sync(0xffffffffu, cs[x], 8);
                    cs[x] += __shfl_xor_sync(0xffffffffu, cs[x], 16);
                    if (g == 0) colsum[((second ? 4 : 0) + tb) * 64 + j0 + x] = cs[x];
                }
            }
        }
        // the products with the states, scaled by token, and their dot products with q and k
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
            const int r = 16 * tb + g + 8 * hh;
            const float sq = a.scale * G.ec[r], sr = -G.ec[r] * G.beta[r], st = G.tail[r] * G.beta[r];
            float dot[3] = {};
#pragma unroll
            for (int j = 0; j < HT; ++j) {
                const float2 qv = sQ.get2(r, col0 + 8 * j + 2 * t), kv = sK.get2(r, col0 + 8 * j + 2 * t);
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    float &eq = dq[j][2 * hh + x], &er = dkr[j][2 * hh + x];
                    const float et = dkt[j][2 * hh + x] * st, kx = x ? kv.y : kv.x;
                    eq *= sq;
                    er *= sr;
                    dot[0] = fmaf(x ? qv.y : qv.x, eq, dot[0]);
                    dot[1] = fmaf(kx, er, dot[1]);
                    dot[2] = fmaf(kx, et, dot[2]);
                    er += et;
                }
            }
#pragma unroll
            for (int x = 0; x < 3; ++x) {
                dot[x] += __shfl_xor_sync(0xffffffffu, dot[x], 1);
                dot[x] += __shfl_xor_sync(0xffffffffu, dot[x], 2);
                if (t == 0) dots[(qt * 3 + x) * 64 + r] = dot[x];
            }
            rs[hh] += __shfl_xor_sync(0xffffffffu, rs[hh], 1);
            rs[hh] += __shfl_xor_sync(0xffffffffu, rs[hh], 2);
            if (t == 0) rowsum[qt * 64 + r] = rs[hh];
        }
        {
            constexpr int per = N / 64;
            float v = bdot.x + bdot.y;
#pragma unroll
            for (int d = 1; d < per; d <<= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
            if (tid % per == 0) dbeta[tid / per] = v;
            v = sdot.x + sdot.y;
#pragma unroll
            for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
            if (lane == 0) blocks[w] = v;
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            FragA<T, sizeof(T) == 2 ? 2 : 1> fp, fa;
            FragB<T, 1> b0, b1;
            if (j <= tb) {
                sDP.a_mk(fp, 16 * tb, 16 * j);
                sDA.a_mk(fa, 16 * tb, 16 * j);
#pragma unroll
                for (int d = 0; d < HT / 2; ++d) {
                    sK.b_kn(b0, b1, 16 * j, col0 + 16 * d);
                    mma16(dq[2 * d], fp, b0);
                    mma16(dq[2 * d + 1], fp, b1);
                    mma16(dkr[2 * d], fa, b0);
                    mma16(dkr[2 * d + 1], fa, b1);
                }
            }
            if (j >= tb) {
                sDP.a_km(fp, 16 * tb, 16 * j);
                sDA.a_km(fa, 16 * tb, 16 * j);
#pragma unroll
                for (int d = 0; d < HT / 2; ++d) {
                    sK.b_kn(b0, b1, 16 * j, col0 + 16 * d);
                    mma16(dkr[2 * d], fa, b0);
                    mma16(dkr[2 * d + 1], fa, b1);
                    sQ.b_kn(b0, b1, 16 * j, col0 + 16 * d);
                    mma16(dkr[2 * d], fp, b0);
                    mma16(dkr[2 * d + 1], fp, b1);
                }
            }
        }
        if (w == 0) {
            // dg: the suffix sums of `suf`, the prefix sums (before t) of `pre`, and the chunk's own decay
            float suf[2], pre[2], ds = 0.0f;
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const int r = 2 * lane + x;
                float cs = 0.0f, up = 0.0f, dn = 0.0f;
#pragma unroll
                for (int j = 0; j < 8; ++j) cs += colsum[j * 64 + r];
#pragma unroll
                for (int j = 0; j < NG; ++j) {
                    up += rowsum[j * 64 + r] + (dots[j * 192 + r] + dots[j * 192 + 64 + r]);
                    dn += dots[j * 192 + 128 + r];
                }
                suf[x] = up - cs;
                pre[x] = dn;
            }
#pragma unroll
            for (int j = 0; j < SM::warps; ++j) ds += blocks[j];
            float sfx = suf[0] + suf[1], p = pre[0] + pre[1];
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const float s2 = __shfl_down_sync(0xffffffffu, sfx, d), p2 = __shfl_up_sync(0xffffffffu, p, d);
                if (lane + d < 32) sfx += s2;
                if (lane >= d) p += p2;
            }
            p -= pre[0] + pre[1];  // before this lane's tokens
            const float tail = G.last * ds;
            T *dgp = (T*)a.dg + tok * a.Hv + h, *dbp = (T*)a.dbeta + tok * a.Hv + h;
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const int r = 2 * lane + x;
                if (r >= n) continue;
                dgp[(long long)r * a.Hv] = io<T>::to((x ? sfx - suf[0] : sfx) + (x ? p + pre[0] : p) + tail);
                dbp[(long long)r * a.Hv] = io<T>::to(dbeta[r]);
            }
        }
        // out: to the sums of the head's group, or (the last of it) to dq and dk
        const bool part = !SM::totals && share > 1, done = i + 1 == steps;
        if (SM::totals && share > 1) {
#pragma unroll
            for (int hh = 0; hh < 2; ++hh)
#pragma unroll
                for (int j = 0; j < HT; ++j) {
                    const int r = 16 * tb + g + 8 * hh, cc = col0 + 8 * j + 2 * t;
                    float2 *tq = reinterpret_cast<float2*>(tot + r * DK + cc), *tk = reinterpret_cast<float2*>(tot + (64 + r) * DK + cc);
                    if (i >= vslices) {  // (this thread's own places)
                        dq[j][2 * hh] += tq->x, dq[j][2 * hh + 1] += tq->y;
                        dkr[j][2 * hh] += tk->x, dkr[j][2 * hh + 1] += tk->y;
                    }
                    if (!done) {
                        *tq = make_float2(dq[j][2 * hh], dq[j][2 * hh + 1]);
                        *tk = make_float2(dkr[j][2 * hh], dkr[j][2 * hh + 1]);
                    }
                }
        }
        if (done || part) {
            const bool vec = a.Dk % 8 == 0 && ((reinterpret_cast<uintptr_t>(a.dq) | reinterpret_cast<uintptr_t>(a.dk)) & 15) == 0;
#pragma unroll
            for (int hh = 0; hh < 2; ++hh) {
                const int r = 16 * tb + g + 8 * hh;
                const long long row = ((tok + r) * a.Hk + hk) * a.Dk;
                if (part) {
                    float* to = c.part + ((tok + r) * a.Hv + h) * 2 * a.Dk;
#pragma unroll
                    for (int j = 0; j < HT; ++j)
#pragma unroll
                        for (int x = 0; x < 2; ++x) {
                            const int cc = col0 + 8 * j + 2 * t + x;
                            if (r < n && cc < a.Dk) to[cc] = dq[j][2 * hh + x], to[a.Dk + cc] = dkr[j][2 * hh + x];
                        }
                } else if (vec) {
                    if constexpr (sizeof(T) == 2) {
                        static_assert(HT == 4, "the four lanes of a row store a tile each");
#pragma unroll
                        for (int y = 0; y < 2; ++y) {
                            uint32_t v[4];
#pragma unroll
                            for (int j = 0; j < 4; ++j)
                                v[j] = y ? pack_bf16(dkr[j][2 * hh], dkr[j][2 * hh + 1]) : pack_bf16(dq[j][2 * hh], dq[j][2 * hh + 1]);
                            quad_transpose(v);
                            const int cc = col0 + 8 * t;
                            if (r < n && cc < a.Dk) *reinterpret_cast<uint4*>((T*)(y ? a.dk : a.dq) + row + cc) = make_uint4(v[0], v[1], v[2], v[3]);
                        }
                    } else {
#pragma unroll
                        for (int j = 0; j < HT; ++j) {
                            const int cc = col0 + 8 * j + 2 * t;
                            if (r >= n || cc >= a.Dk) continue;
                            *reinterpret_cast<float2*>((T*)a.dq + row + cc) = make_float2(dq[j][2 * hh], dq[j][2 * hh + 1]);
                            *reinterpret_cast<float2*>((T*)a.dk + row + cc) = make_float2(dkr[j][2 * hh], dkr[j][2 * hh + 1]);
                        }
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < HT; ++j)
#pragma unroll
                        for (int x = 0; x < 2; ++x) {
                            const int cc = col0 + 8 * j + 2 * t + x;
                            if (r >= n || cc >= a.Dk) continue;
                            ((T*)a.dq)[row + cc] = io<T>::to(dq[j][2 * hh + x]);
                            ((T*)a.dk)[row + cc] = io<T>::to(dkr[j][2 * hh + x]);
                        }
                }
            }
        }
        if (!done) {
            __syncthreads();  // dP, dA and the sums have been read
            if (!SM::ahead) load(i + 1);
        }
    }
}

template <typename T, int DK>
vmb_status launch_grad_dk(const DeltaGrad& c, cudaStream_t stream) {
    using SM = GradSmem<T, DK>;
    const void* fn = (const void*)delta_grad_kernel<T, DK>;
    const long long grid = (long long)c.a.B * (SM::totals ? c.a.Hk : c.a.Hv) * chunks_of(c.a.T);
    if (!allow_smem(fn, SM::total)) return VMB_ERR_CUDA;
    DeltaGrad arg = c;
    void* args[] = {&arg};
    return launch_kernel(fn, dim3((unsigned)grid), dim3(SM::threads), SM::total, args, stream) == cudaSuccess ? VMB_OK : VMB_ERR_CUDA;
}

// Whether the value heads of a key head leave their dq and dk to be summed by delta_share_kernel.
static_assert(GradSmem<float, 64>::totals && GradSmem<__nv_bfloat16, 64>::totals && GradSmem<__nv_bfloat16, 128>::totals, "sums in the CTA");
inline bool grad_leaves_parts(const DeltaArgs& a) { return a.Hv != a.Hk && a.dtype == VMB_F32 && a.Dk > 64 && !GradSmem<float, 128>::totals; }

template <typename T>
vmb_status launch_grad(const DeltaGrad& c, cudaStream_t stream) {
    return c.a.Dk <= 64 ? launch_grad_dk<T, 64>(c, stream) : launch_grad_dk<T, 128>(c, stream);
}

}  // namespace vmb
