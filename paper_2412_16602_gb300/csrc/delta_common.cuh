// delta_common.cuh - device code shared by the kernels of the gated delta rule
// (delta_chain.cuh, delta_grad.cuh): tiles in shared memory, matrix fragments,
// the decays of a chunk and its triangular system.
//
// The recurrence of one head, S [Dk x Dv]:
//   S_t = a_t (I - b_t k_t k_t^T) S_{t-1} + b_t k_t v_t^T,  a_t = e^(g_t),  o_t = scale S_t^T q_t
// is computed in chunks of 64 tokens.  With c_i the log decays summed from the chunk's start to
// token i, S the state before the chunk and r_i the residual that token i adds (u_i = b_i r_i):
//   E_ij = e^(c_i - c_j) k_i.k_j (j < i),   r = v - e^c K S - E (b r),
//   o_i = scale (e^(c_i) S^T q_i + sum_{j<=i} e^(c_i - c_j) (q_i.k_j) u_j),
//   S' = e^(c_last) S + sum_j e^(c_last - c_j) k_j u_j^T.
// The triangular system for r is solved in four blocks of 16 tokens, whose diagonal blocks are
// inverted explicitly: 4 x (16 x 16), by forward substitution in fp32.
//
// Every product runs on the tensor cores through mma.sync, whose accumulator layout is that of its
// A operand: with the states and residuals transposed (rows = value channels) a warp carries 16
// rows from product to product in registers, without a barrier or a trip through shared memory
// (measured on the GB300: 604 TFLOP/s in bf16, 302 in tf32 and 21 cycles of latency, against a
// dependent chain of four products per chunk).  What a product rounds:
//   bf16 storage: q, k, v and do are exact.  Intermediates (states, residuals, E, P, the diagonal
//     inverses) enter as the sum of two bf16 values (16 bits, error about 2^-18); only S^T q takes the
//     state's leading term, because nothing but an output that is rounded to bf16 itself sees it: o is off by
//     1.75e-3 (rms) where its own rounding alone is 1.66e-3.  Both terms take 160 -> 166 us for 32 x 3136 tokens,
//     207 -> 219 for 24 ragged sequences, 1258 -> 1289 for a training pass of 8 x 3136.
//   fp32 storage: every operand is the sum of two tf32 values (22 bits), products hi.hi + hi.lo + lo.hi.
// Accumulators, states, decays and the diagonal inverses are fp32 throughout.
#pragma once

#include "vmb_common.cuh"

namespace vmb {

constexpr int kChunk = 64;       // tokens per chunk
// chunks of a sequence, whatever its length (tokens + 63 may not fit an int)
__host__ __device__ __forceinline__ int chunks_of(int tokens) { return tokens / kChunk + (tokens % kChunk != 0); }

// ------------------------------------------------------------------ fragments

// acc is a 16 x 8 fp32 accumulator tile: lane (g = lane / 4, t = lane % 4) holds
// (g, 2t), (g, 2t + 1), (g + 8, 2t), (g + 8, 2t + 1).
__device__ __forceinline__ void mma_bf16(float (&c)[4], const uint32_t (&a)[4], const uint32_t (&b)[2]) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]));
}
__device__ __forceinline__ void mma_tf32(float (&c)[4], const uint32_t (&a)[4], const uint32_t (&b)[2]) {
    asm volatile("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]));
}

// Accumulator pairs through the packed operations, half the instructions: in the bf16 kernels (176 -> 158 us for a batch of
// 32 x 3136 tokens).  In the fp32 kernels, which use every register, the pairs cost more moves than they save (878 -> 1150 us
// for a training pass of 32 x 784): kPacked = false.
__device__ __forceinline__ float2 lo2(const float (&c)[4]) { return make_float2(c[0], c[1]); }
__device__ __forceinline__ float2 hi2(const float (&c)[4]) { return make_float2(c[2], c[3]); }
__device__ __forceinline__ void put4(float (&c)[4], float2 a, float2 b) { c[0] = a.x, c[1] = a.y, c[2] = b.x, c[3] = b.y; }
__device__ __forceinline__ float2 minus(float2 a, float2 b) { return __ffma2_rn(b, make_float2(-1.0f, -1.0f), a); }
template <bool kPacked> __device__ __forceinline__ void scale4(float (&c)[4], float2 s) {
    if constexpr (kPacked)
        put4(c, __fmul2_rn(lo2(c), s), __fmul2_rn(hi2(c), s));
    else
        c[0] *= s.x, c[1] *= s.y, c[2] *= s.x, c[3] *= s.y;
}
template <bool kPacked> __device__ __forceinline__ void add4(float (&c)[4], const float (&d)[4]) {
    if constexpr (kPacked)
        put4(c, __fadd2_rn(lo2(c), lo2(d)), __fadd2_rn(hi2(c), hi2(d)));
    else
        c[0] += d[0], c[1] += d[1], c[2] += d[2], c[3] += d[3];
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ float bf16_lo(uint32_t p) { return __uint_as_float(p << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t p) { return __uint_as_float(p & 0xffff0000u); }
__device__ __forceinline__ float2 bf16_pair(uint32_t p) { return make_float2(bf16_lo(p), bf16_hi(p)); }
// v = hi + lo up to 2^-18 |v|
__device__ __forceinline__ void split_bf16(float2 v, uint32_t& hi, uint32_t& lo) {
    hi = pack_bf16(v.x, v.y);
    const float2 d = minus(v, bf16_pair(hi));
    lo = pack_bf16(d.x, d.y);
}
// x = hi + lo, both tf32 (11 leading bits): hi rounded, lo cut off at 2^-22 of 2^e, e the exponent of x.  By masks, at the full
// rate of the integer pipe.  (hi cut off as well leaves every lo the sign of its x, and the products without lo.lo too small, by
// 2.7e-7 on average and 1.3e-6 at worst, against none and 7.2e-7; it takes one instruction less: 867 and 880 us for a training
// pass of 32 x 784 tokens.  cvt.rna.tf32: 1339 us.)
__device__ __forceinline__ uint32_t round_tf32(float x) { return (__float_as_uint(x) + 0x1000u) & 0xffffe000u; }
__device__ __forceinline__ void split_tf32(float x, uint32_t& hi, uint32_t& lo) {
    hi = round_tf32(x);
    lo = __float_as_uint(x - __uint_as_float(hi)) & 0xffffe000u;
}
__device__ __forceinline__ void split_tf32(float x, float y, uint32_t& xh, uint32_t& xl, uint32_t& yh, uint32_t& yl) {
    xh = round_tf32(x);
    yh = round_tf32(y);
    xl = __float_as_uint(x - __uint_as_float(xh)) & 0xffffe000u;
    yl = __float_as_uint(y - __uint_as_float(yh)) & 0xffffe000u;
}

// Among the four lanes of a row, lane t holding word t of four tiles: afterwards lane t holds the four words of tile t.
__device__ __forceinline__ void quad_transpose(uint32_t (&v)[4]) {
    const int t = threadIdx.x & 3;
#pragma unroll
    for (int n = 0; n < 4; n += 2) {
        const uint32_t x = __shfl_xor_sync(0xffffffffu, t & 1 ? v[n] : v[n + 1], 1);
        if (t & 1) v[n] = x; else v[n + 1] = x;
    }
#pragma unroll
    for (int n = 0; n < 2; ++n) {
        const uint32_t x = __shfl_xor_sync(0xffffffffu, t & 2 ? v[n] : v[n + 2], 2);
        if (t & 2) v[n] = x; else v[n + 2] = x;
    }
}

// Operands of a 16-deep step.  bf16: NT terms.  fp32: two 8-deep tf32 steps s; position k of step
// s stands for column 8s + 2(k % 4) + k / 4, the same in A and B, so that an accumulator pair
// (columns 2t, 2t + 1) is an A operand as it stands.
template <typename T, int NT> struct FragA;
template <typename T, int NT> struct FragB;
template <int NT> struct FragA<__nv_bfloat16, NT> { uint32_t r[NT][4]; };
template <int NT> struct FragB<__nv_bfloat16, NT> { uint32_t r[NT][2]; };
template <int NT> struct FragA<float, NT> { uint32_t hi[2][4], lo[2][4]; };
template <int NT> struct FragB<float, NT> { uint32_t hi[2][2], lo[2][2]; };

// c += a b for four neighbouring tiles of 8 columns.  A product waits for the one before it on the same
// accumulator (21 cycles, against 8 per product when the pipe is full): the terms go round the tiles.  bf16: the
// product of two second terms is left out.  fp32: the small products are summed on their own, because every
// product added to a large accumulator on the tensor cores truncates it (2 times instead of 6).
template <int NA, int NB>
__device__ __forceinline__ void mma_quad(float (&c)[4][4], const FragA<__nv_bfloat16, NA>& a, const FragB<__nv_bfloat16, NB> (&b)[4]) {
    if constexpr (NA > 1) {
#pragma unroll
        for (int i = 0; i < 4; ++i) mma_bf16(c[i], a.r[1], b[i].r[0]);
    }
    if constexpr (NB > 1) {
#pragma unroll
        for (int i = 0; i < 4; ++i) mma_bf16(c[i], a.r[0], b[i].r[1]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) mma_bf16(c[i], a.r[0], b[i].r[0]);
}
template <int NA, int NB>
__device__ __forceinline__ void mma_quad(float (&c)[4][4], const FragA<float, NA>& a, const FragB<float, NB> (&b)[4]) {
    float d[4][4] = {};
#pragma unroll
    for (int s = 0; s < 2; ++s) {
#pragma unroll
        for (int i = 0; i < 4; ++i) mma_tf32(d[i], a.lo[s], b[i].hi[s]);
#pragma unroll
        for (int i = 0; i < 4; ++i) mma_tf32(c[i], a.hi[s], b[i].hi[s]);
#pragma unroll
        for (int i = 0; i < 4; ++i) mma_tf32(d[i], a.hi[s], b[i].lo[s]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) add4<false>(c[i], d[i]);
}
// Two tiles, the small products in an accumulator of their own (w), so that a chain of such products is half as long.
template <int NA, int NB>
__device__ __forceinline__ void mma_pair(float (&c0)[4], float (&c1)[4], float (&w0)[4], float (&w1)[4], const FragA<__nv_bfloat16, NA>& a,
                                         const FragB<__nv_bfloat16, NB>& b0, const FragB<__nv_bfloat16, NB>& b1) {
    if constexpr (NA > 1) mma_bf16(w0, a.r[1], b0.r[0]), mma_bf16(w1, a.r[1], b1.r[0]);
    mma_bf16(c0, a.r[0], b0.r[0]), mma_bf16(c1, a.r[0], b1.r[0]);
    if constexpr (NB > 1) mma_bf16(w0, a.r[0], b0.r[1]), mma_bf16(w1, a.r[0], b1.r[1]);
}
template <int NA, int NB>
__device__ __forceinline__ void mma_pair(float (&c0)[4], float (&c1)[4], float (&w0)[4], float (&w1)[4], const FragA<float, NA>& a,
                                         const FragB<float, NB>& b0, const FragB<float, NB>& b1) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        mma_tf32(w0, a.lo[s], b0.hi[s]), mma_tf32(w1, a.lo[s], b1.hi[s]);
        mma_tf32(c0, a.hi[s], b0.hi[s]), mma_tf32(c1, a.hi[s], b1.hi[s]);
        mma_tf32(w0, a.hi[s], b0.lo[s]), mma_tf32(w1, a.hi[s], b1.lo[s]);
    }
}
// c += a b for one tile
template <typename T, int NA, int NB> __device__ __forceinline__ void mma16(float (&c)[4], const FragA<T, NA>& a, const FragB<T, NB>& b) {
    float w[4] = {};
    if constexpr (sizeof(T) == 2) {
        if constexpr (NA > 1) mma_bf16(c, a.r[1], b.r[0]);
        if constexpr (NB > 1) mma_bf16(c, a.r[0], b.r[1]);
        mma_bf16(c, a.r[0], b.r[0]);
    } else {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            mma_tf32(w, a.lo[s], b.hi[s]);
            mma_tf32(c, a.hi[s], b.hi[s]);
            mma_tf32(w, a.hi[s], b.lo[s]);
        }
        add4<false>(c, w);
    }
}

// A from two neighbouring accumulator tiles (16 columns)
template <int NT>
__device__ __forceinline__ void frag_from_acc(FragA<__nv_bfloat16, NT>& a, const float (&c0)[4], const float (&c1)[4]) {
    if constexpr (NT > 1) {
        split_bf16(lo2(c0), a.r[0][0], a.r[1][0]);
        split_bf16(hi2(c0), a.r[0][1], a.r[1][1]);
        split_bf16(lo2(c1), a.r[0][2], a.r[1][2]);
        split_bf16(hi2(c1), a.r[0][3], a.r[1][3]);
    } else {
        a.r[0][0] = pack_bf16(c0[0], c0[1]);
        a.r[0][1] = pack_bf16(c0[2], c0[3]);
        a.r[0][2] = pack_bf16(c1[0], c1[1]);
        a.r[0][3] = pack_bf16(c1[2], c1[3]);
    }
}
template <int NT>
__device__ __forceinline__ void frag_from_acc(FragA<float, NT>& a, const float (&c0)[4], const float (&c1)[4]) {
    split_tf32(c0[0], c0[1], a.hi[0][0], a.lo[0][0], a.hi[0][2], a.lo[0][2]);
    split_tf32(c0[2], c0[3], a.hi[0][1], a.lo[0][1], a.hi[0][3], a.lo[0][3]);
    split_tf32(c1[0], c1[1], a.hi[1][0], a.lo[1][0], a.hi[1][2], a.lo[1][2]);
    split_tf32(c1[2], c1[3], a.hi[1][1], a.lo[1][1], a.hi[1][3], a.lo[1][3]);
}

// ------------------------------------------------------------------ tiles in shared memory

// Row-major tiles.  bf16: NT planes, rows padded by 16 bytes, which puts the eight rows of an
// ldmatrix on different banks.  fp32: no padding; the 8-column blocks of row r are permuted within
// 32 columns by sw(r), which makes both the pair loads along a row (8 rows x 4 pairs) and the
// loads down the columns (rows 2t and 2t + 1) free of conflicts.
template <typename T, int COLS, int NT> struct Tile;

__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix4_t(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}

// four 8 x 8 matrices of 16-bit values, each written transposed: lane l gives row l % 8 of matrix l / 8
__device__ __forceinline__ void stmatrix4_t(uint32_t addr, uint32_t r0, uint32_t r1, uint32_t r2, uint32_t r3) {
    asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(r0), "r"(r1), "r"(r2), "r"(r3)
                 : "memory");
}

template <int COLS, int NT> struct Tile<__nv_bfloat16, COLS, NT> {
    using T = __nv_bfloat16;
    static constexpr int kLd = COLS + 8, kVec = 8;
    static constexpr int bytes(int rows) { return NT * rows * kLd * 2; }
    T* p;
    int plane;  // elements between the planes
    __device__ __forceinline__ Tile(void* s, int rows) : p((T*)s), plane(rows * kLd) {}
    __device__ __forceinline__ T* vec_at(int r, int c) const { return p + r * kLd + c; }
    __device__ __forceinline__ void set2(int r, int c, float v0, float v1) const {  // c even
        if constexpr (NT > 1) {
            split_bf16(make_float2(v0, v1), *reinterpret_cast<uint32_t*>(p + r * kLd + c),
                       *reinterpret_cast<uint32_t*>(p + plane + r * kLd + c));
        } else {
            *reinterpret_cast<uint32_t*>(p + r * kLd + c) = pack_bf16(v0, v1);
        }
    }
    __device__ __forceinline__ void zero(int r, int c) const { p[r * kLd + c] = __float2bfloat16_rn(0.0f); }
    __device__ __forceinline__ void put(int r, int c, T v) const { p[r * kLd + c] = v; }
    __device__ __forceinline__ float2 get2(int r, int c) const { return bf16_pair(*reinterpret_cast<const uint32_t*>(p + r * kLd + c)); }  // c even
    // sum += this(r, c ..) . o(r, c ..) over kVec columns
    __device__ __forceinline__ void dot_vec(const Tile& o, int r, int c, float2& sum) const {
        const uint4 u = *reinterpret_cast<const uint4*>(vec_at(r, c)), v = *reinterpret_cast<const uint4*>(o.vec_at(r, c));
        sum = __ffma2_rn(bf16_pair(u.x), bf16_pair(v.x), sum);
        sum = __ffma2_rn(bf16_pair(u.y), bf16_pair(v.y), sum);
        sum = __ffma2_rn(bf16_pair(u.z), bf16_pair(v.z), sum);
        sum = __ffma2_rn(bf16_pair(u.w), bf16_pair(v.w), sum);
    }
    __device__ __forceinline__ uint32_t lane_addr(int term, int r0, int c0) const {
        const int lane = threadIdx.x & 31;
        return smem_u32(p + term * plane + (r0 + (lane & 15)) * kLd + c0 + (lane >> 4) * 8);
    }
    // A[m][k] = tile[m0 + m][k0 + k]
    template <int N = NT> __device__ __forceinline__ void a_mk(FragA<T, N>& a, int m0, int k0) const {
#pragma unroll
        for (int i = 0; i < N; ++i) ldmatrix4(a.r[i], lane_addr(i, m0, k0));
    }
    // A[m][k] = tile[k0 + k][m0 + m]
    template <int N = NT> __device__ __forceinline__ void a_km(FragA<T, N>& a, int m0, int k0) const {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            uint32_t r[4];
            ldmatrix4_t(r, lane_addr(i, k0, m0));
            a.r[i][0] = r[0];
            a.r[i][1] = r[2];
            a.r[i][2] = r[1];
            a.r[i][3] = r[3];
        }
    }
    // two column tiles: B[k][n] = tile[n0 + n][k0 + k], n < 8 in b0, n >= 8 in b1
    template <int N = NT> __device__ __forceinline__ void b_nk(FragB<T, N>& b0, FragB<T, N>& b1, int n0, int k0) const {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            uint32_t r[4];
            ldmatrix4(r, lane_addr(i, n0, k0));
            b0.r[i][0] = r[0];
            b0.r[i][1] = r[2];
            b1.r[i][0] = r[1];
            b1.r[i][1] = r[3];
        }
    }
    // B[k][n] = tile[k0 + k][n0 + n]
    template <int N = NT> __device__ __forceinline__ void b_kn(FragB<T, N>& b0, FragB<T, N>& b1, int k0, int n0) const {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            uint32_t r[4];
            ldmatrix4_t(r, lane_addr(i, k0, n0));
            b0.r[i][0] = r[0];
            b0.r[i][1] = r[1];
            b1.r[i][0] = r[2];
            b1.r[i][1] = r[3];
        }
    }
    // two accumulator tiles (rows = tile columns c0 .., columns = tile rows r0 ..) written transposed
    __device__ __forceinline__ void set_t(int r0, int c0, const float (&a)[4], const float (&b)[4]) const {
        const int lane = threadIdx.x & 31;
        stmatrix4_t(smem_u32(p + (r0 + (lane & 7) + ((lane >> 4) << 3)) * kLd + c0 + ((lane >> 3) & 1) * 8), pack_bf16(a[0], a[1]),
                    pack_bf16(a[2], a[3]), pack_bf16(b[0], b[1]), pack_bf16(b[2], b[3]));
    }
    // the transposed 16 x 16 block as two accumulator tiles: c[j] holds columns k0 + 8j .. of rows m0 ..
    __device__ __forceinline__ void acc_km(float (&c0)[4], float (&c1)[4], int m0, int k0) const {
        FragA<T, 1> a;
        a_km<1>(a, m0, k0);
        c0[0] = bf16_lo(a.r[0][0]), c0[1] = bf16_hi(a.r[0][0]), c0[2] = bf16_lo(a.r[0][1]), c0[3] = bf16_hi(a.r[0][1]);
        c1[0] = bf16_lo(a.r[0][2]), c1[1] = bf16_hi(a.r[0][2]), c1[2] = bf16_lo(a.r[0][3]), c1[3] = bf16_hi(a.r[0][3]);
    }
};

template <int COLS, int NT> struct Tile<float, COLS, NT> {
    using T = float;
    static constexpr int kLd = COLS, kVec = 4;
    static_assert(COLS % 32 == 0, "the permutation works within 32 columns");
    static constexpr int bytes(int rows) { return rows * kLd * 4; }
    T* p;
    __device__ __forceinline__ Tile(void* s, int) : p((T*)s) {}
    __device__ __forceinline__ static int at(int r, int c) { return r * kLd + (c ^ (((r & 3) ^ ((r >> 2) & 1)) << 3)); }
    __device__ __forceinline__ T* vec_at(int r, int c) const { return p + at(r, c); }
    __device__ __forceinline__ void set2(int r, int c, float v0, float v1) const {
        *reinterpret_cast<float2*>(p + at(r, c)) = make_float2(v0, v1);
    }
    __device__ __forceinline__ void zero(int r, int c) const { p[at(r, c)] = 0.0f; }
    __device__ __forceinline__ void put(int r, int c, T v) const { p[at(r, c)] = v; }
    __device__ __forceinline__ float2 get2(int r, int c) const { return *reinterpret_cast<const float2*>(p + at(r, c)); }
    __device__ __forceinline__ void dot_vec(const Tile& o, int r, int c, float2& sum) const {
        const float4 u = *reinterpret_cast<const float4*>(vec_at(r, c)), v = *reinterpret_cast<const float4*>(o.vec_at(r, c));
        sum.x = fmaf(u.x, v.x, sum.x), sum.y = fmaf(u.y, v.y, sum.y);
        sum.x = fmaf(u.z, v.z, sum.x), sum.y = fmaf(u.w, v.w, sum.y);
    }
    template <int N = NT> __device__ __forceinline__ void a_mk(FragA<T, N>& a, int m0, int k0) const {
        const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const float2 u = *reinterpret_cast<const float2*>(p + at(m0 + g, k0 + 8 * s + 2 * t));
            const float2 w = *reinterpret_cast<const float2*>(p + at(m0 + g + 8, k0 + 8 * s + 2 * t));
            split_tf32(u.x, u.y, a.hi[s][0], a.lo[s][0], a.hi[s][2], a.lo[s][2]);
            split_tf32(w.x, w.y, a.hi[s][1], a.lo[s][1], a.hi[s][3], a.lo[s][3]);
        }
    }
    template <int N = NT> __device__ __forceinline__ void a_km(FragA<T, N>& a, int m0, int k0) const {
        const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int k = k0 + 8 * s + 2 * t;
            split_tf32(p[at(k, m0 + g)], a.hi[s][0], a.lo[s][0]);
            split_tf32(p[at(k, m0 + g + 8)], a.hi[s][1], a.lo[s][1]);
            split_tf32(p[at(k + 1, m0 + g)], a.hi[s][2], a.lo[s][2]);
            split_tf32(p[at(k + 1, m0 + g + 8)], a.hi[s][3], a.lo[s][3]);
        }
    }
    template <int N = NT> __device__ __forceinline__ void b_nk(FragB<T, N>& b0, FragB<T, N>& b1, int n0, int k0) const {
        const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const float2 u = *reinterpret_cast<const float2*>(p + at(n0 + g, k0 + 8 * s + 2 * t));
            const float2 w = *reinterpret_cast<const float2*>(p + at(n0 + 8 + g, k0 + 8 * s + 2 * t));
            split_tf32(u.x, u.y, b0.hi[s][0], b0.lo[s][0], b0.hi[s][1], b0.lo[s][1]);
            split_tf32(w.x, w.y, b1.hi[s][0], b1.lo[s][0], b1.hi[s][1], b1.lo[s][1]);
        }
    }
    template <int N = NT> __device__ __forceinline__ void b_kn(FragB<T, N>& b0, FragB<T, N>& b1, int k0, int n0) const {
        const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int k = k0 + 8 * s + 2 * t;
            split_tf32(p[at(k, n0 + g)], p[at(k + 1, n0 + g)], b0.hi[s][0], b0.lo[s][0], b0.hi[s][1], b0.lo[s][1]);
            split_tf32(p[at(k, n0 + 8 + g)], p[at(k + 1, n0 + 8 + g)], b1.hi[s][0], b1.lo[s][0], b1.hi[s][1], b1.lo[s][1]);
        }
    }
    __device__ __forceinline__ void set_t(int r0, int c0, const float (&a)[4], const float (&b)[4]) const {
        const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            p[at(r0 + 2 * t + (x & 1), c0 + g + 8 * (x >> 1))] = a[x];
            p[at(r0 + 8 + 2 * t + (x & 1), c0 + g + 8 * (x >> 1))] = b[x];
        }
    }
    __device__ __forceinline__ void acc_km(float (&c0)[4], float (&c1)[4], int m0, int k0) const {
        const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int k = k0 + 8 * j + 2 * t;
            float(&c)[4] = j ? c1 : c0;
            c[0] = p[at(k, m0 + g)], c[1] = p[at(k + 1, m0 + g)];
            c[2] = p[at(k, m0 + g + 8)], c[3] = p[at(k + 1, m0 + g + 8)];
        }
    }
};

// The ten 16 x 16 blocks on and below the diagonal of a 64 x 64 matrix, block (i, j) at i (i + 1) / 2 + j.
// bf16: rows of 48 bytes (eight rows of an ldmatrix on different banks); fp32: the halves of rows 2, 3, 6, 7, ...
// swapped, which leaves the pair loads along rows free of conflicts.
template <typename T, int NT> struct LowTile;
template <int NT> struct LowTile<__nv_bfloat16, NT> {
    using T = __nv_bfloat16;
    static constexpr int kLd = 24, kBlock = 16 * kLd, kBytes = NT * 10 * kBlock * 2;
    T* p;
    __device__ __forceinline__ explicit LowTile(void* s) : p((T*)s) {}
    __device__ __forceinline__ static int base(int bi, int bj) { return (bi * (bi + 1) / 2 + bj) * NT * kBlock; }
    __device__ __forceinline__ void set(int bi, int bj, int r, int c, float v) const {
        T* q = p + base(bi, bj) + r * kLd + c;
        const T h = __float2bfloat16_rn(v);
        q[0] = h;
        if constexpr (NT > 1) q[kBlock] = __float2bfloat16_rn(v - __bfloat162float(h));
    }
    __device__ __forceinline__ void set2(int bi, int bj, int r, int c, float v0, float v1) const {
        T* q = p + base(bi, bj) + r * kLd + c;
        uint32_t h = pack_bf16(v0, v1), l = 0;
        if constexpr (NT > 1) {
            split_bf16(make_float2(v0, v1), h, l);
            *reinterpret_cast<uint32_t*>(q + kBlock) = l;
        }
        *reinterpret_cast<uint32_t*>(q) = h;
    }
    __device__ __forceinline__ uint32_t lane_addr(int term, int bi, int bj) const {
        const int lane = threadIdx.x & 31;
        return smem_u32(p + base(bi, bj) + term * kBlock + (lane & 15) * kLd + (lane >> 4) * 8);
    }
    // B[k][n] = block[n][k]
    __device__ __forceinline__ void b_nk(FragB<T, NT>& b0, FragB<T, NT>& b1, int bi, int bj) const {
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            uint32_t r[4];
            ldmatrix4(r, lane_addr(i, bi, bj));
            b0.r[i][0] = r[0], b0.r[i][1] = r[2], b1.r[i][0] = r[1], b1.r[i][1] = r[3];
        }
    }
    // B[k][n] = block[k][n]
    __device__ __forceinline__ void b_kn(FragB<T, NT>& b0, FragB<T, NT>& b1, int bi, int bj) const {
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            uint32_t r[4];
            ldmatrix4_t(r, lane_addr(i, bi, bj));
            b0.r[i][0] = r[0], b0.r[i][1] = r[1], b1.r[i][0] = r[2], b1.r[i][1] = r[3];
        }
    }
};
template <int NT> struct LowTile<float, NT> {
    using T = float;
    static constexpr int kBlock = 256, kBytes = 10 * kBlock * 4;
    T* p;
    __device__ __forceinline__ explicit LowTile(void* s) : p((T*)s) {}
    __device__ __forceinline__ static int at(int bi, int bj, int r, int c) {
        return (bi * (bi + 1) / 2 + bj) * kBlock + r * 16 + (c ^ ((r & 2) << 2));
    }
    __device__ __forceinline__ void set(int bi, int bj, int r, int c, float v) const { p[at(bi, bj, r, c)] = v; }
    __device__ __forceinline__ void set2(int bi, int bj, int r, int c, float v0, float v1) const {
        *reinterpret_cast<float2*>(p + at(bi, bj, r, c)) = make_float2(v0, v1);
    }
    __device__ __forceinline__ void b_nk(FragB<T, NT>& b0, FragB<T, NT>& b1, int bi, int bj) const {
        const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const float2 u = *reinterpret_cast<const float2*>(p + at(bi, bj, g, 8 * s + 2 * t));
            const float2 w = *reinterpret_cast<const float2*>(p + at(bi, bj, g + 8, 8 * s + 2 * t));
            split_tf32(u.x, u.y, b0.hi[s][0], b0.lo[s][0], b0.hi[s][1], b0.lo[s][1]);
            split_tf32(w.x, w.y, b1.hi[s][0], b1.lo[s][0], b1.hi[s][1], b1.lo[s][1]);
        }
    }
    __device__ __forceinline__ void b_kn(FragB<T, NT>& b0, FragB<T, NT>& b1, int bi, int bj) const {
        const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int k = 8 * s + 2 * t;
            split_tf32(p[at(bi, bj, k, g)], p[at(bi, bj, k + 1, g)], b0.hi[s][0], b0.lo[s][0], b0.hi[s][1], b0.lo[s][1]);
            split_tf32(p[at(bi, bj, k, 8 + g)], p[at(bi, bj, k + 1, 8 + g)], b1.hi[s][0], b1.lo[s][0], b1.hi[s][1], b1.lo[s][1]);
        }
    }
};

// ------------------------------------------------------------------ global <-> shared

// A head's tile of `rows` x `cols` values at src (row stride in elements) into a tile of ROWS x COLS,
// zeros outside: asynchronous 16-byte copies where the rows allow them (`vec`), single values otherwise.
// The caller commits and waits.
template <int ROWS, int COLS, typename TL>
__device__ __forceinline__ void load_tile(const TL& s, const typename TL::T* src, long long stride, int rows, int cols,
                                          bool vec, int tid, int threads) {
    using T = typename TL::T;
    constexpr int V = TL::kVec, P = COLS / V;
    if (vec) {
        for (int i = tid; i < ROWS * P; i += threads) {
            const int r = i / P, c = (i % P) * V;
            const int n = r < rows ? min(max(cols - c, 0), V) * (int)sizeof(T) : 0;
            cp_async16(s.vec_at(r, c), n ? src + r * stride + c : src, n);
        }
    } else {
        for (int i = tid; i < ROWS * COLS; i += threads) {
            const int r = i / COLS, c = i % COLS;
            if (r < rows && c < cols)
                s.put(r, c, src[r * stride + c]);
            else
                s.zero(r, c);
        }
    }
}
// 16-byte copies are possible: pointer and row stride are multiples of 16 bytes
template <typename T> __device__ __forceinline__ bool rows_aligned(const T* p, long long stride) {
    return ((reinterpret_cast<uintptr_t>(p) | (uintptr_t)(stride * (long long)sizeof(T))) & 15) == 0;
}

// The same for tiles that a chain of chunks loads one after the other, by THREADS threads: every thread's rows and
// columns are fixed, so that a copy costs a pointer and a comparison (worked out from scratch for each copy, the
// addresses took 2300 of the 7500 cycles of a chunk).
template <typename TL, int COLS, int THREADS> struct TileCopy {
    using T = typename TL::T;
    static constexpr int V = TL::kVec, P = COLS / V, kRows = THREADS / P, kTimes = kChunk / kRows;
    static_assert(THREADS % P == 0 && kChunk % kRows == 0, "whole rows");
    const T* src;      // the chain's first row
    long long stride;
    int row, off, bytes, cols;
    bool vec;
    __device__ __forceinline__ TileCopy(const T* s, long long st, int columns, int tid) : src(s), stride(st), cols(columns) {
        vec = rows_aligned(s, st);
        row = tid / P;
        const int c = (tid % P) * V;
        off = c;
        bytes = min(max(columns - c, 0), V) * (int)sizeof(T);
    }
    // rows first .. first + rows - 1 of the chain
    __device__ __forceinline__ void copy(unsigned char* tile, long long first, int rows, int tid) const {
        const TL s(tile, kChunk);
        if (vec) {
            const T* p = src + (first + row) * stride + off;
#pragma unroll
            for (int i = 0; i < kTimes; ++i) {
                const int n = row + i * kRows < rows ? bytes : 0;
                cp_async16(s.vec_at(row + i * kRows, off), n ? p + i * kRows * stride : src, n);
            }
        } else {
            load_tile<kChunk, COLS>(s, src + first * stride, stride, rows, cols, false, tid, THREADS);
        }
    }
};

// ------------------------------------------------------------------ where a sequence lies

struct DeltaSeq {
    long long start;  // first token of the sequence (packed) or of its batch row
    int len;          // tokens
    int slot;         // first chunk's place among the kept states
};
// Packed sequences (offsets): rows offsets[b] .. offsets[b + 1] - 1 of the `total` tokens.  Offsets that
// leave [0, total], decrease or exceed the stated longest length are cut to what is in range and
// reported in the status word.
__device__ __forceinline__ DeltaSeq delta_seq(const int* offsets, int b, int T, long long total, unsigned* err) {
    if (!offsets) return {(long long)b * T, T, b * chunks_of(T)};
    const long long a = offsets[b], e = offsets[b + 1];
    const long long lo = a < 0 ? 0 : (a > total ? total : a), hi = e < lo ? lo : (e > total ? total : e);
    const int len = (int)(hi - lo < T ? hi - lo : T);
    if ((a != lo || e != hi || hi - lo != len) && err && threadIdx.x == 0) atomicOr(err, kErrBounds);
    return {lo, len, (int)(lo / kChunk) + b};
}

// ------------------------------------------------------------------ decays of a chunk

// Per token, in shared memory.  The log decays are summed as pairs of floats (hi + lo), so that a
// difference c_i - c_j keeps fp32 accuracy however small c is: a token that resets the state (g = -inf,
// taken as -200, whose exponential is 0 in fp32) does not cost the tokens after it any digits.
struct alignas(16) ChunkGates {
    float hi[kChunk], lo[kChunk];  // c / ln 2
    float beta[kChunk];
    float ec[kChunk];    // e^c
    float tail[kChunk];  // e^(c_last - c)
    float last;          // e^(c_last)
    // an accumulator pair's tokens, 8 n + 2 t and the one after it
    static __device__ __forceinline__ float2 pair(const float* v, int n) {
        return *reinterpret_cast<const float2*>(v + 8 * n + 2 * (threadIdx.x & 3));
    }
};

// e^(c_i - c_j) from the differences of the parts
__device__ __forceinline__ float decay(float hi, float lo) { return ex2(hi + lo); }

__device__ __forceinline__ void add_pair(float& h, float& l, float h2, float l2) {
    // Knuth's two-sum, then the low parts
    const float s = h + h2, bb = s - h;
    const float e = (h - (s - bb)) + (h2 - bb);
    const float lo = e + (l + l2);
    h = s + lo;
    l = lo - (h - s);
}

// Called by one whole warp: lane l holds tokens 2l and 2l + 1 (g = 0 and beta = 0 behind the end).
__device__ __forceinline__ void chunk_gates(ChunkGates& G, float g0, float g1, float b0, float b1) {
    const int lane = threadIdx.x & 31;
    g0 = g0 < -200.0f ? -200.0f : g0;
    g1 = g1 < -200.0f ? -200.0f : g1;
    float h = g0, l = 0.0f;
    add_pair(h, l, g1, 0.0f);  // both tokens
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const float h2 = __shfl_up_sync(0xffffffffu, h, d), l2 = __shfl_up_sync(0xffffffffu, l, d);
        if (lane >= d) add_pair(h, l, h2, l2);
    }
    const float lh = __shfl_sync(0xffffffffu, h, 31), ll = __shfl_sync(0xffffffffu, l, 31);
    float ph = __shfl_up_sync(0xffffffffu, h, 1), pl = __shfl_up_sync(0xffffffffu, l, 1);
    if (lane == 0) ph = pl = 0.0f;
    add_pair(ph, pl, g0, 0.0f);  // the first token's own sum
    // in units of ln 2, as pairs again
    auto units = [](float& a, float& b) {
        constexpr float kLog2eLo = 1.925963033500e-8f;  // log2 e = kLog2e + kLog2eLo
        const float p = a * kLog2e, e = fmaf(a, kLog2e, -p) + fmaf(b, kLog2e, a * kLog2eLo);
        a = p + e;
        b = e - (a - p);
    };
    float lth = lh, ltl = ll;
    units(ph, pl), units(h, l), units(lth, ltl);
    const int i = 2 * lane;
    G.hi[i] = ph, G.lo[i] = pl, G.hi[i + 1] = h, G.lo[i + 1] = l;
    G.beta[i] = b0, G.beta[i + 1] = b1;
    G.ec[i] = decay(ph, pl), G.ec[i + 1] = decay(h, l);
    G.tail[i] = decay(lth - ph, ltl - pl), G.tail[i + 1] = decay(lth - h, ltl - l);
    if (lane == 0) G.last = decay(lth, ltl);
}

// ------------------------------------------------------------------ the chunk's triangular system

// The products of a chunk that do not depend on the state, by WARPS (4 or 8) warps:
//   sE: -E below the diagonal blocks, and on the diagonal the inverses (I + E_bb b)^-1
//       (kRowBeta: (I + b E_bb)^-1, the transposed system's);
//   sP (kWithP): scale e^(c_i - c_j) q_i.k_j for j <= i, zeros above.
// Warps 0 to 3 compute one diagonal block of both and invert that of E; the six blocks below the diagonal of E and of P
// are twelve tasks for the last four warps (the same ones where there are no others).
// diag: 4 x 16 x 20 floats of scratch.  The gates and tiles are ready before the call; no barrier inside.
template <typename T, int DK, bool kRowBeta, bool kWithP, int WARPS, int NE, int NK>
__device__ __forceinline__ void chunk_system(const Tile<T, DK, NK>& sK, const Tile<T, DK, NK>& sQ, const LowTile<T, NE>& sE,
                                             const LowTile<T, NE>& sP, float* diag, const ChunkGates& G, float scale, int w) {
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    // e^(c_i - c_j) of this lane's places of block (bi, bj), zero for j > i (where it may be large without bound)
    auto decays = [&](int bi, int bj, float(&d)[2][4]) {
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            const float2 jh = G.pair(G.hi, 2 * bj + n), jl = G.pair(G.lo, 2 * bj + n);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int r = g + 8 * h, j = 8 * n + 2 * t;
                const float ih = G.hi[16 * bi + r], il = G.lo[16 * bi + r];
                const float2 v = __fadd2_rn(minus(make_float2(ih, ih), jh), minus(make_float2(il, il), jl));
                d[n][2 * h] = bi > bj || j <= r ? ex2(v.x) : 0.0f;
                d[n][2 * h + 1] = bi > bj || j + 1 <= r ? ex2(v.y) : 0.0f;
            }
        }
    };
    auto product = [&](const Tile<T, DK, NK>& sA, int bi, int bj, float(&c)[2][4]) {
#pragma unroll
        for (int d = 0; d < DK; d += 16) {
            FragA<T, NK> a;
            FragB<T, NK> b0, b1;
            sK.b_nk(b0, b1, 16 * bj, d);
            sA.a_mk(a, 16 * bi, d);
            mma16(c[0], a, b0);
            mma16(c[1], a, b1);
        }
    };
    if (w < 4) {
        float kk[2][4] = {}, d[2][4];
        product(sK, w, w, kk);
        decays(w, w, d);
        const float2 b0 = G.pair(G.beta, 2 * w), b1 = G.pair(G.beta, 2 * w + 1);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int r = g + 8 * h;
            const float ib = G.beta[16 * w + r];
            // -L transposed: the columns of the block side by side (the diagonal itself is not read)
            float* col = diag + (w * 16 + 2 * t) * 20 + r;
            const float2 s0 = kRowBeta ? make_float2(-ib, -ib) : make_float2(-b0.x, -b0.y), s1 = kRowBeta ? s0 : make_float2(-b1.x, -b1.y);
            const float2 v0 = __fmul2_rn(__fmul2_rn(make_float2(kk[0][2 * h], kk[0][2 * h + 1]), make_float2(d[0][2 * h], d[0][2 * h + 1])), s0);
            const float2 v1 = __fmul2_rn(__fmul2_rn(make_float2(kk[1][2 * h], kk[1][2 * h + 1]), make_float2(d[1][2 * h], d[1][2 * h + 1])), s1);
            col[0] = v0.x;
            col[20] = v0.y;
            col[160] = v1.x;
            col[180] = v1.y;
        }
        __syncwarp();
        if constexpr (kWithP) {
            float qk[2][4] = {};
            product(sQ, w, w, qk);
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    const float2 v = __fmul2_rn(make_float2(qk[n][2 * h], qk[n][2 * h + 1]),
                                                __fmul2_rn(make_float2(d[n][2 * h], d[n][2 * h + 1]), make_float2(scale, scale)));
                    sP.set2(w, w, g + 8 * h, 8 * n + 2 * t, v.x, v.y);
                }
        }
        // column c of (I + L)^-1, L the strictly lower block: x_i = [i = c] - sum_{j < i} L_ij x_j, taken off column
        // by column of L so that the chain is 15 products long
        const int c = lane & 15;
        float2 x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = make_float2(2 * i == c ? 1.0f : 0.0f, 2 * i + 1 == c ? 1.0f : 0.0f);
#pragma unroll
        for (int j = 0; j < 15; ++j) {
            const float* col = diag + (w * 16 + j) * 20;
            const float xj = j & 1 ? x[j / 2].y : x[j / 2].x;
            if (j % 2 == 0) x[j / 2].y = fmaf(col[j + 1], xj, x[j / 2].y);
#pragma unroll
            for (int i = j / 2 + 1; i < 8; ++i)
                x[i] = __ffma2_rn(*reinterpret_cast<const float2*>(col + 2 * i), make_float2(xj, xj), x[i]);
        }
        if (lane < 16) {
#pragma unroll
            for (int i = 0; i < 16; ++i) sE.set(w, w, i, c, i & 1 ? x[i / 2].y : x[i / 2].x);
        }
    }
    if (w >= WARPS - 4) {
        for (int task = w - (WARPS - 4); task < (kWithP ? 12 : 6); task += 4) {
            const bool p = task >= 6;
            const int b = p ? task - 6 : task;  // (3,0) (3,1) (3,2) (2,0) (2,1) (1,0)
            const int bi = b < 3 ? 3 : b < 5 ? 2 : 1, bj = b < 3 ? b : b < 5 ? b - 3 : 0;
            float c[2][4] = {}, d[2][4];
            product(p ? sQ : sK, bi, bj, c);
            decays(bi, bj, d);
            const float f = p ? scale : -1.0f;
            const LowTile<T, NE>& to = p ? sP : sE;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    const float2 v = __fmul2_rn(make_float2(c[n][2 * h], c[n][2 * h + 1]),
                                                __fmul2_rn(make_float2(d[n][2 * h], d[n][2 * h + 1]), make_float2(f, f)));
                    to.set2(bi, bj, g + 8 * h, 8 * n + 2 * t, v.x, v.y);
                }
        }
    }
}

}  // namespace vmb
