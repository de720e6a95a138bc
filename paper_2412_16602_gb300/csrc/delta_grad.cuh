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
// One CTA per chunk and value head, eight warps: warp w computes the 16 tokens of block w % 4 for one half
// of the Dk columns, and of the 64 x 64 products dP (first half) or dA (second).  The value channels come
// in slices of 64.  Scales by token are applied to the accumulators, so that the operands are the kept
// values themselves.
#pragma once

#include "delta_common.cuh"
#include "delta_internal.h"

namespace vmb {

constexpr int kGradThreads = 256;

template <typename T, int DK> struct GradSmem {
    using KT = Tile<T, DK, 1>;
    using VT = Tile<T, 64, 1>;
    using PT = Tile<T, 64, sizeof(T) == 2 ? 2 : 1>;
    static constexpr int k = 0, q = k + KT::bytes(64), d = q + KT::bytes(64), r = d + VT::bytes(64), x = r + VT::bytes(64),
                         s = x + VT::bytes(64), ds = s + KT::bytes(64), tiles = ds + KT::bytes(64);
    // dP and dA take the place of do .. dS
    static constexpr int dp = d, da = dp + PT::bytes(64);
    static_assert(da + PT::bytes(64) <= tiles, "dP and dA fit");
    static constexpr int gates = tiles, sums = gates + (int)sizeof(ChunkGates);
    // row sums [2][64], column sums [2][4][64], dots [2][3][64], dbeta [64], block sums [8]
    static constexpr int total = sums + 4 * (128 + 512 + 384 + 64 + 8);
};

template <typename T, int DK>
__global__ void __launch_bounds__(kGradThreads) delta_grad_kernel(DeltaGrad c) {
    using SM = GradSmem<T, DK>;
    constexpr int HT = DK / 16;  // column tiles of 8 per warp
    extern __shared__ __align__(128) unsigned char smem[];
    const DeltaArgs& a = c.a;
    const int tid = threadIdx.x, w = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    const int tb = w & 3, hf = w >> 2, col0 = hf * (DK / 2);
    pdl_launch_dependents();
    pdl_wait();
    const int chunks = (a.T + kChunk - 1) / kChunk;
    const int ch = blockIdx.x % chunks;
    const long long chain = blockIdx.x / chunks;
    const int h = (int)(chain % a.Hv), b = (int)(chain / a.Hv);
    const DeltaSeq seq = delta_seq(a.offsets, b, a.T, a.total, c.err);
    const int n = min(seq.len - ch * kChunk, kChunk);
    if (n <= 0) return;

    const int hk = h / (a.Hv / a.Hk);
    const long long brow = a.offsets ? 0 : b, tok0 = (a.offsets ? seq.start : 0) + (long long)ch * kChunk;
    const long long tok = seq.start + (long long)ch * kChunk;  // in the dense tensors
    const T* kp = (const T*)a.k + brow * a.k_b + tok0 * a.k_t + (long long)hk * a.Dk;
    const T* qp = (const T*)a.q + brow * a.q_b + tok0 * a.q_t + (long long)hk * a.Dk;
    const long long hrow = (long long)a.Hv * a.Dv, off = tok * hrow + (long long)h * a.Dv;
    const T *dp = (const T*)a.dout + off, *rp = (const T*)a.saved_r + off, *xp = (const T*)c.dx + off;
    const long long srow = ((long long)(seq.slot + ch) * a.Hv + h) * a.Dv * a.Dk;
    const T *sp = (const T*)a.saved + srow, *dsp = (const T*)c.ds + srow;

    const typename SM::KT sK(smem + SM::k, 64), sQ(smem + SM::q, 64), sS(smem + SM::s, 64), sDS(smem + SM::ds, 64);
    const typename SM::VT sD(smem + SM::d, 64), sR(smem + SM::r, 64), sX(smem + SM::x, 64);
    const typename SM::PT sDP(smem + SM::dp, 64), sDA(smem + SM::da, 64);
    ChunkGates& G = *reinterpret_cast<ChunkGates*>(smem + SM::gates);
    float* rowsum = reinterpret_cast<float*>(smem + SM::sums);
    float *colsum = rowsum + 128, *dots = colsum + 512, *dbeta = dots + 384, *blocks = dbeta + 64;

    load_tile<64, DK>(sK, kp, a.k_t, n, a.Dk, rows_aligned(kp, a.k_t), tid, kGradThreads);
    load_tile<64, DK>(sQ, qp, a.q_t, n, a.Dk, rows_aligned(qp, a.q_t), tid, kGradThreads);
    if (w == 0) {
        const T *gp = (const T*)a.g + tok * a.Hv + h, *bp = (const T*)a.beta + tok * a.Hv + h;
        float v[4];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            v[i] = 2 * lane + i < n ? io<T>::cvt(gp[(long long)(2 * lane + i) * a.Hv]) : 0.0f;
            v[2 + i] = 2 * lane + i < n ? io<T>::cvt(bp[(long long)(2 * lane + i) * a.Hv]) : 0.0f;
        }
        chunk_gates(G, v[0], v[1], v[2], v[3]);
    }

    float dq[HT][4] = {}, dkr[HT][4] = {}, dkt[HT][4] = {}, W[8][4] = {};
    float sdot = 0.0f, bdot = 0.0f;
    for (int v0 = 0; v0 < a.Dv; v0 += 64) {
        const int cols = min(a.Dv - v0, 64);
        if (v0) __syncthreads();
        load_tile<64, 64>(sD, dp + v0, hrow, n, cols, rows_aligned(dp + v0, hrow), tid, kGradThreads);
        load_tile<64, 64>(sR, rp + v0, hrow, n, cols, rows_aligned(rp + v0, hrow), tid, kGradThreads);
        load_tile<64, 64>(sX, xp + v0, hrow, n, cols, rows_aligned(xp + v0, hrow), tid, kGradThreads);
        const T *s0 = sp + (long long)v0 * a.Dk, *ds0 = dsp + (long long)v0 * a.Dk;
        load_tile<64, DK>(sS, s0, a.Dk, cols, a.Dk, rows_aligned(s0, a.Dk), tid, kGradThreads);
        load_tile<64, DK>(sDS, ds0, a.Dk, cols, a.Dk, rows_aligned(ds0, a.Dk), tid, kGradThreads);
        cp_async_commit();
        cp_async_wait<0>();
        __syncthreads();
        {  // this thread's part of dbeta: token tid / 4, every fourth channel
            const int i = tid >> 2, q4 = tid & 3;
#pragma unroll 4
            for (int j = 0; j < 16; ++j) bdot = fmaf(sX.get(i, q4 + 4 * j), sR.get(i, q4 + 4 * j), bdot);
            for (int j = tid; j < 64 * DK; j += kGradThreads) sdot = fmaf(sS.get(j / DK, j % DK), sDS.get(j / DK, j % DK), sdot);
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
            for (int j = 0; j < 4; ++j)
                if (j <= tb) {
                    sR.b_nk(b0, b1, 16 * j, 16 * kk);
                    mma16(W[2 * j], hf ? fx : fd, b0);
                    mma16(W[2 * j + 1], hf ? fx : fd, b1);
                }
        }
    }
    // dP or dA, and their products with q k^T or k k^T
    {
        float m[8][4] = {};
#pragma unroll
        for (int d = 0; d < DK / 16; ++d) {
            FragA<T, 1> f;
            FragB<T, 1> b0, b1;
            if (hf) sK.a_mk(f, 16 * tb, 16 * d); else sQ.a_mk(f, 16 * tb, 16 * d);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (j <= tb) {
                    sK.b_nk(b0, b1, 16 * j, 16 * d);
                    mma16(m[2 * j], f, b0);
                    mma16(m[2 * j + 1], f, b1);
                }
        }
        __syncthreads();  // do, r, dX, S and dS have been read
        float rs[2] = {};
#pragma unroll
        for (int jt = 0; jt < 8; ++jt) {
            float cs[2] = {};
            if (jt / 2 <= tb) {
#pragma unroll
                for (int hh = 0; hh < 2; ++hh) {
                    const int i = 16 * tb + g + 8 * hh;
                    float v[2];
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const int j = 8 * jt + 2 * t + x;
                        const float e = j <= i ? decay(G.hi[i] - G.hi[j], G.lo[i] - G.lo[j]) * G.beta[j] : 0.0f;
                        const float f = hf ? (j < i ? -e * G.beta[i] : 0.0f) : a.scale * e;
                        v[x] = f * W[jt][2 * hh + x];
                        const float p = v[x] * m[jt][2 * hh + x];
                        rs[hh] += p;
                        cs[x] += p;
                    }
                    (hf ? sDA : sDP).set2(i, 8 * jt + 2 * t, v[0], v[1]);
                }
            }
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                cs[x] += __shfl_xor_sync(0xffffffffu, cs[x], 4);
                cs[x] += __shfl_xor_sync(0xffffffffu, cs[x], 8);
                cs[x] += __shfl_xor_sync(0xffffffffu, cs[x], 16);
                if (g == 0) colsum[(hf * 4 + tb) * 64 + 8 * jt + 2 * t + x] = cs[x];
            }
        }
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
            rs[hh] += __shfl_xor_sync(0xffffffffu, rs[hh], 1);
            rs[hh] += __shfl_xor_sync(0xffffffffu, rs[hh], 2);
            if (t == 0) rowsum[hf * 64 + 16 * tb + g + 8 * hh] = rs[hh];
        }
    }
    // the products with the states, scaled by token, and their dot products with q and k
#pragma unroll
    for (int hh = 0; hh < 2; ++hh) {
        const int i = 16 * tb + g + 8 * hh;
        const float sq = a.scale * G.ec[i], sr = -G.ec[i] * G.beta[i], st = G.tail[i] * G.beta[i];
        float dot[3] = {};
#pragma unroll
        for (int j = 0; j < HT; ++j)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const int cc = col0 + 8 * j + 2 * t + x;
                const float qv = sQ.get(i, cc), kv = sK.get(i, cc);
                float &eq = dq[j][2 * hh + x], &er = dkr[j][2 * hh + x];
                const float et = dkt[j][2 * hh + x] * st;
                eq *= sq;
                er *= sr;
                dot[0] = fmaf(qv, eq, dot[0]);
                dot[1] = fmaf(kv, er, dot[1]);
                dot[2] = fmaf(kv, et, dot[2]);
                er += et;
            }
#pragma unroll
        for (int x = 0; x < 3; ++x) {
            dot[x] += __shfl_xor_sync(0xffffffffu, dot[x], 1);
            dot[x] += __shfl_xor_sync(0xffffffffu, dot[x], 2);
            if (t == 0) dots[(hf * 3 + x) * 64 + i] = dot[x];
        }
    }
    bdot += __shfl_xor_sync(0xffffffffu, bdot, 1);
    bdot += __shfl_xor_sync(0xffffffffu, bdot, 2);
    if ((tid & 3) == 0) dbeta[tid >> 2] = bdot;
#pragma unroll
    for (int d = 16; d; d >>= 1) sdot += __shfl_xor_sync(0xffffffffu, sdot, d);
    if (lane == 0) blocks[w] = sdot;
    __syncthreads();

#pragma unroll
    for (int j = 0; j < 4; ++j) {
        FragA<T, sizeof(T) == 2 ? 2 : 1> fp, fa, fpt, fat;
        const bool low = j <= tb, high = j >= tb;
        if (low) sDP.a_mk(fp, 16 * tb, 16 * j), sDA.a_mk(fa, 16 * tb, 16 * j);
        if (high) sDP.a_km(fpt, 16 * tb, 16 * j), sDA.a_km(fat, 16 * tb, 16 * j);
        FragB<T, 1> b0, b1;
#pragma unroll
        for (int d = 0; d < HT / 2; ++d) {
            sK.b_kn(b0, b1, 16 * j, col0 + 16 * d);
            if (low) {
                mma16(dq[2 * d], fp, b0);
                mma16(dq[2 * d + 1], fp, b1);
                mma16(dkr[2 * d], fa, b0);
                mma16(dkr[2 * d + 1], fa, b1);
            }
            if (high) {
                mma16(dkr[2 * d], fat, b0);
                mma16(dkr[2 * d + 1], fat, b1);
                sQ.b_kn(b0, b1, 16 * j, col0 + 16 * d);
                mma16(dkr[2 * d], fpt, b0);
                mma16(dkr[2 * d + 1], fpt, b1);
            }
        }
    }
    const bool shared = a.Hv != a.Hk;
#pragma unroll
    for (int hh = 0; hh < 2; ++hh) {
        const int i = 16 * tb + g + 8 * hh;
        if (i >= n) continue;
        const long long row = shared ? ((tok + i) * a.Hv + h) * 2 * a.Dk : ((tok + i) * a.Hk + hk) * a.Dk;
#pragma unroll
        for (int j = 0; j < HT; ++j)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const int cc = col0 + 8 * j + 2 * t + x;
                if (cc >= a.Dk) continue;
                if (shared) {
                    c.part[row + cc] = dq[j][2 * hh + x];
                    c.part[row + a.Dk + cc] = dkr[j][2 * hh + x];
                } else {
                    ((T*)a.dq)[row + cc] = io<T>::to(dq[j][2 * hh + x]);
                    ((T*)a.dk)[row + cc] = io<T>::to(dkr[j][2 * hh + x]);
                }
            }
    }
    if (w == 0) {
        // dg: the suffix sums of `suf`, the prefix sums (before t) of `pre`, and the chunk's own decay
        float suf[2], pre[2], ds = 0.0f;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int i = 2 * lane + x;
            float cs = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) cs += colsum[j * 64 + i];
            suf[x] = (rowsum[i] + rowsum[64 + i] - cs) + (dots[i] + dots[192 + i]) + (dots[64 + i] + dots[256 + i]);
            pre[x] = dots[128 + i] + dots[320 + i];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) ds += blocks[i];
        float s = suf[0] + suf[1], p = pre[0] + pre[1];
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const float s2 = __shfl_down_sync(0xffffffffu, s, d), p2 = __shfl_up_sync(0xffffffffu, p, d);
            if (lane + d < 32) s += s2;
            if (lane >= d) p += p2;
        }
        p -= pre[0] + pre[1];  // before this lane's tokens
        const float tail = G.last * ds;
        T *dgp = (T*)a.dg + tok * a.Hv + h, *dbp = (T*)a.dbeta + tok * a.Hv + h;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int i = 2 * lane + x;
            if (i >= n) continue;
            dgp[(long long)i * a.Hv] = io<T>::to((x ? s - suf[0] : s) + (x ? p + pre[0] : p) + tail);
            dbp[(long long)i * a.Hv] = io<T>::to(dbeta[i]);
        }
    }
}

template <typename T, int DK>
vmb_status launch_grad_dk(const DeltaGrad& c, cudaStream_t stream) {
    const void* fn = (const void*)delta_grad_kernel<T, DK>;
    const long long grid = (long long)c.a.B * c.a.Hv * ((c.a.T + kChunk - 1) / kChunk);
    const size_t smem = GradSmem<T, DK>::total;
    if (cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) return VMB_ERR_CUDA;
    DeltaGrad arg = c;
    void* args[] = {&arg};
    return launch_kernel(fn, dim3((unsigned)grid), dim3(kGradThreads), smem, args, stream) == cudaSuccess ? VMB_OK : VMB_ERR_CUDA;
}

template <typename T>
vmb_status launch_grad(const DeltaGrad& c, cudaStream_t stream) {
    return c.a.Dk <= 64 ? launch_grad_dk<T, 64>(c, stream) : launch_grad_dk<T, 128>(c, stream);
}

}  // namespace vmb
