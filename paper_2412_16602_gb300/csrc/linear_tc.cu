// linear_tc.cu - the matrix product on the fifth-generation tensor cores: out [M][N] = epilogue(A B^T), A and B with the contraction
// dense (forward: x and the weights) or with their rows dense (gradients: dx takes the weights so, dW both operands).
//
// Tiles of 256 x 256 by a pair of CTAs (each holds half of the rows of A and of B in its shared memory and 128 x 256 sums in its
// tensor memory), or of 128 x 128 by one CTA where those would leave SMs idle.  One warp starts tensor copies into a ring of stages
// of 128 bytes of the contraction, swizzled by 128 bytes; one thread of the pair issues the products; eight warps take the sums of one buffer of
// tensor memory through the epilogue while the products of the next tile go to the other.  Where tiles are few and the contraction long
// it is split, the parts' sums are kept in fp32 and joined in order by a second launch.
//
// 8192^3 in bf16: 582 us, 1889 TFLOP/s (the library's product 542); 16384 x 1536 x 6144 in bf16 183 (165), in e4m3 102 to 109, with SiLU 113, with GELU 140.  Long contractions are
// bound by the products and by the bytes into an SM alike (32 KB and 512 clocks a stage); short ones by the epilogue, whose two warps on each
// scheduler wait for their own results in turn (0.39 instructions a clock): with a quarter of the products issued that last case takes the same.
// Tried: outputs by tensor copies from shared memory (130 without GELU, 173 with it: each needs a proxy fence), sixteen warps (96 registers: 128 and 156), factors and biases
// asked for a tile ahead (no change), four stages of the ring (8192^3 652).  Arrivals at the pair's barrier carry no release at the cluster's scope: what they
// order are tensor-memory reads, by the tcgen05 fences; with it a warp waited for its stores (151 with GELU).
// Every wait is bounded; one that gives up leaves kErrTimeout in the workspace's header and ends the kernel.
#include <cuda.h>
#include <cudaTypedefs.h>

#include <mutex>

#include "linear_common.cuh"
#include "vmb_testing.h"

namespace vmb {

namespace {

constexpr int kTcEpiWarps = 8, kTcThreads = 32 * (2 + kTcEpiWarps), kTcStages = 5;
constexpr int kTcA = 128 * 128;  // bytes of A in a stage, and of B: 128 rows of 128 bytes of the contraction
constexpr int kTcStage = 2 * kTcA;
constexpr int kTcEpiBytes = 4096 + 1024;  // of each warp of the epilogue: 32 x 64 outputs on their way, factors and biases of 128 columns
constexpr int kTcSmem = 1024 + kTcStages * kTcStage + kTcEpiWarps * kTcEpiBytes;

struct TcKernel {
    CUtensorMap ta, tb;
    GemmEpilogue e;
    float* partial;  // [splits][M][N]
    unsigned* err;
    long long M;
    int N;
    int tiles_m, tiles_n, splits, kblocks, kper, units;
    bool vec;
    bool drop;  // test hook: the sums of a CTA's first unit are not handed over, so every wait for them runs out
};

// Tensor-memory matrix descriptors of operands swizzled by 128 bytes.  The contraction dense: rows of 128 bytes, eight rows every 1024
// bytes, a step of 32 bytes along the contraction moves the start.  The rows dense: 64 rows every 128 x 64 bytes, eight steps of the
// contraction every 1024.
__device__ __forceinline__ uint64_t tc_desc(uint32_t addr, bool rows_dense) {
    const uint64_t lead = rows_dense ? (8192 >> 4) : 1;
    return (uint64_t)((addr >> 4) & 0x3FFF) | lead << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}

// fp32 sums of bf16 (or e4m3) A and B; bits 15 and 16: rows dense.
template <int CG, int BN, bool kBits8, bool kArow, bool kBrow> constexpr uint32_t tc_idesc() {
    return (1u << 4) | (kBits8 ? 0u : 1u << 7 | 1u << 10) | (kArow ? 1u << 15 : 0u) | (kBrow ? 1u << 16 : 0u) | (uint32_t)(BN >> 3) << 17 |
           (uint32_t)((128 * CG) >> 4) << 24;
}

template <int CG, bool kBits8> __device__ __forceinline__ void tc_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t add) {
    if constexpr (CG == 2 && kBits8)
        asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n}\n" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(add));
    else if constexpr (CG == 2)
        asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(add));
    else if constexpr (kBits8)
        asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n}\n" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(add));
    else
        asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(add));
}

// The products issued so far arrive at `bar` of every CTA of the pair when they are done.
template <int CG> __device__ __forceinline__ void tc_commit(uint32_t bar) {
    if constexpr (CG == 2) {
        const uint16_t both = 3;
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"(both) : "memory");
    } else {
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
    }
}

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t in_first_cta(uint32_t addr) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(addr));
    return r;
}
__device__ __forceinline__ void cluster_barrier() {
    asm volatile("barrier.cluster.arrive.aligned;\n barrier.cluster.wait.aligned;" ::: "memory");
}

// A box of the map from (x, y) into this CTA's shared memory; its bytes count at `bar`, which may be the first CTA's.
template <int CG> __device__ __forceinline__ void tc_load(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
    if constexpr (CG == 2)
        asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
                     "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(bar)
                     : "memory");
    else
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
                     "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(bar)
                     : "memory");
}

// (the sums of a tile may take long: kTcSumsNs)
constexpr uint64_t kTcSumsNs = 4ull * 1000 * 1000 * 1000;
__device__ __forceinline__ bool tc_wait(uint32_t bar, uint32_t parity, unsigned* err, uint64_t limit = kWaitLimitNs) {
    if (mbarrier_wait(bar, parity, limit)) return true;
    atomicOr(err, kErrTimeout);
    return false;
}

// 32 columns of the warp's 32 lanes; they are there after tmem_wait32.
__device__ __forceinline__ void tmem_load32(uint32_t (&r)[32], uint32_t addr) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,"
        "%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
          "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]),
          "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr));
}
__device__ __forceinline__ void tmem_wait32(uint32_t (&r)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]),
                   "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]),
                   "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
                 :
                 : "memory");
}

struct TcUnit {
    int m, n, split;
};
// Units in order: the parts of a tile, then tiles down the rows within bands of 16 (the band's rows of A and all of B pass through the L2 cache once).
__device__ __forceinline__ TcUnit tc_unit(const TcKernel& k, int u) {
    TcUnit t;
    t.split = u % k.splits;
    const int tile = u / k.splits, band = tile / (16 * k.tiles_n), in = tile - band * 16 * k.tiles_n;
    const int high = min(16, k.tiles_m - band * 16);
    t.m = band * 16 + in % high;
    t.n = in / high;
    return t;
}

// The rows and columns that a warp has of a unit; a lane's row.
struct TcRows {
    int m0, n0, split;
    bool on;
    long long at;  // of the row's first column in the output
    float scale;
};

template <int ACT> __device__ __forceinline__ void activate_pairs(float2 (&v)[16]) {
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = activate2<ACT>(v[i]);
}
__device__ __forceinline__ uint32_t bf16_pair(float2 v) {
    const __nv_bfloat162 p = __float22bfloat162_rn(v);
    return *reinterpret_cast<const uint32_t*>(&p);
}

// The sums of 32 columns of a lane's row, from column c of its warp's on, with their factors and bias.
template <int COLS> __device__ __forceinline__ void tc_scale(const TcKernel& k, float2 (&v)[16], const TcRows& t, int c, const uint32_t (&r)[32], const float* terms) {
    const float2 rs = make_float2(t.scale, t.scale);
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        const float4 b = *reinterpret_cast<const float4*>(terms + COLS + c + 4 * q);
        v[2 * q] = make_float2(__uint_as_float(r[4 * q]), __uint_as_float(r[4 * q + 1]));
        v[2 * q + 1] = make_float2(__uint_as_float(r[4 * q + 2]), __uint_as_float(r[4 * q + 3]));
        if (k.e.row_scale) {
            const float4 f = *reinterpret_cast<const float4*>(terms + c + 4 * q);
            v[2 * q] = __ffma2_rn(v[2 * q], __fmul2_rn(make_float2(f.x, f.y), rs), make_float2(b.x, b.y));
            v[2 * q + 1] = __ffma2_rn(v[2 * q + 1], __fmul2_rn(make_float2(f.z, f.w), rs), make_float2(b.z, b.w));
        } else {
            v[2 * q] = __fadd2_rn(v[2 * q], make_float2(b.x, b.y));
            v[2 * q + 1] = __fadd2_rn(v[2 * q + 1], make_float2(b.z, b.w));
        }
    }
}
// A part's sums as they are.
__device__ __forceinline__ void tc_part(const TcKernel& k, const TcRows& t, int c, const uint32_t (&r)[32]) {
    const int n = t.n0 + c;
    float* p = k.partial + (long long)t.split * k.M * k.N + t.at + c;
    if (!t.on) return;
    if (k.vec) {
#pragma unroll
        for (int q = 0; q < 8; ++q)
            if (n + 4 * q < k.N) reinterpret_cast<uint4*>(p)[q] = make_uint4(r[4 * q], r[4 * q + 1], r[4 * q + 2], r[4 * q + 3]);
    } else {
#pragma unroll
        for (int j = 0; j < 32; ++j)
            if (n + j < k.N) p[j] = __uint_as_float(r[j]);
    }
}
// Shared memory: 32 rows of 64 outputs, in pieces of 16 bytes turned by the row: neither a lane for each row nor eight lanes for a row have conflicts.
__device__ __forceinline__ uint4* tc_piece(char* stage, int row, int piece) { return reinterpret_cast<uint4*>(stage + row * 128 + ((piece ^ (row & 7)) << 4)); }
// To (kStore) or from the output's (residual's) rows, eight lanes to a row; n: the first of the 64 columns.
template <bool kStore> __device__ __forceinline__ void tc_rows(const TcKernel& k, __nv_bfloat16* p, const TcRows& t, int n, char* stage) {
    const int lane = threadIdx.x & 31, low = lane >> 3, piece = lane & 7;
    if (n + 8 * piece >= k.N) return;
    p += (long long)(t.m0 + low) * k.N + n + 8 * piece;
    if constexpr (kStore) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (t.m0 + low + 4 * i < k.M) *reinterpret_cast<uint4*>(p + (long long)(4 * i) * k.N) = *tc_piece(stage, low + 4 * i, piece);
    } else {
        uint4 v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (t.m0 + low + 4 * i < k.M) v[i] = *reinterpret_cast<const uint4*>(p + (long long)(4 * i) * k.N);
#pragma unroll
        for (int i = 0; i < 8; ++i) *tc_piece(stage, low + 4 * i, piece) = v[i];
    }
}
// The epilogue of 32 columns of a lane's row, from column c of its warp's on; where the output's rows allow 16 bytes it is left in shared memory, where
// the residual is.
__device__ __forceinline__ void tc_finish(const TcKernel& k, const TcRows& t, int c, float2 (&v)[16], char* stage) {
    const int n = t.n0 + c, lane = threadIdx.x & 31, first = (c & 32) / 8;
    const long long at = t.at + c;
    if (k.e.pre && t.on) {
        if (k.vec) {
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (n + 8 * q < k.N)
                    reinterpret_cast<uint4*>(k.e.pre + at)[q] = make_uint4(bf16_pair(v[4 * q]), bf16_pair(v[4 * q + 1]), bf16_pair(v[4 * q + 2]), bf16_pair(v[4 * q + 3]));
        } else {
#pragma unroll
            for (int j = 0; j < 32; ++j)
                if (n + j < k.N) k.e.pre[at + j] = __float2bfloat16_rn(j & 1 ? v[j / 2].y : v[j / 2].x);
        }
    }
    if (k.e.act == VMB_ACT_SILU) activate_pairs<VMB_ACT_SILU>(v);
    else if (k.e.act == VMB_ACT_GELU) activate_pairs<VMB_ACT_GELU>(v);
    if (!k.vec) {
#pragma unroll
        for (int j = 0; j < 32; ++j)
            if (t.on && n + j < k.N) {
                float y = j & 1 ? v[j / 2].y : v[j / 2].x;
                if (k.e.residual) y += __bfloat162float(k.e.residual[at + j]);
                k.e.out[at + j] = __float2bfloat16_rn(y);
            }
        return;
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        uint4* p = tc_piece(stage, lane, first + q);
        if (k.e.residual) {
            const uint4 r = *p;
            const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) v[4 * q + j] = __fadd2_rn(v[4 * q + j], make_float2(__uint_as_float(w[j] << 16), __uint_as_float(w[j] & 0xffff0000u)));
        }
        *p = make_uint4(bf16_pair(v[4 * q]), bf16_pair(v[4 * q + 1]), bf16_pair(v[4 * q + 2]), bf16_pair(v[4 * q + 3]));
    }
}

template <int CG, int BN, bool kBits8, bool kArow, bool kBrow> __global__ void __launch_bounds__(kTcThreads, 1) gemm_tc_kernel(const __grid_constant__ TcKernel k) {
    static_assert(BN == 128 * CG, "128 rows of B in each CTA");
    constexpr int kCols = 2 * BN, kElems = kBits8 ? 128 : 64;  // columns of tensor memory; elements of the contraction in a stage
    extern __shared__ char smem_raw[];
    __shared__ __align__(8) uint64_t bars[2 * kTcStages + 4];
    __shared__ uint32_t s_tmem;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t rank = CG == 2 ? cluster_rank() : 0;
    const uint32_t base = (smem_u32(smem_raw) + 1023) & ~1023u;
    const uint32_t full = smem_u32(bars), empty = full + 8 * kTcStages, sums_full = empty + 8 * kTcStages, sums_empty = sums_full + 16;
    if (tid == 0) {
        for (int i = 0; i < kTcStages; ++i) mbarrier_init(full + 8 * i, 1), mbarrier_init(empty + 8 * i, 1);
        for (int i = 0; i < 2; ++i) mbarrier_init(sums_full + 8 * i, 1), mbarrier_init(sums_empty + 8 * i, CG * kTcEpiWarps);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (tid == 32 * 3) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&k.ta)) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&k.tb)) : "memory");
    }
    if (warp == 1) {
        if constexpr (CG == 2) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s_tmem)), "n"(kCols));
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s_tmem)), "n"(kCols));
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
        }
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    if constexpr (CG == 2) cluster_barrier();
    else __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = s_tmem;
    pdl_wait();
    pdl_launch_dependents();
    const int first = blockIdx.x / CG, step = gridDim.x / CG;

    if (warp == 0) {
        if (lane == 0) {  // copies
            uint32_t stage = 0, phase = 0;
            bool ok = true;
            for (int u = first; u < k.units && ok; u += step) {
                const TcUnit t = tc_unit(k, u);
                const int m0 = t.m * 128 * CG + (int)rank * 128, n0 = t.n * BN + (int)rank * 128;
                const int kb1 = min(k.kblocks, (t.split + 1) * k.kper);
                for (int kb = t.split * k.kper; kb < kb1; ++kb) {
                    if (!(ok = tc_wait(empty + 8 * stage, phase ^ 1, k.err))) break;
                    const uint32_t a = base + stage * kTcStage, b = a + kTcA;
                    const uint32_t bar = CG == 2 ? in_first_cta(full + 8 * stage) : full + 8 * stage;
                    if (rank == 0) mbarrier_expect_tx(full + 8 * stage, CG * kTcStage);
                    if constexpr (kArow) {
                        tc_load<CG>(a, &k.ta, m0, kb * kElems, bar);
                        tc_load<CG>(a + 8192, &k.ta, m0 + 64, kb * kElems, bar);
                    } else {
                        tc_load<CG>(a, &k.ta, kb * kElems, m0, bar);
                    }
                    if constexpr (kBrow) {
                        tc_load<CG>(b, &k.tb, n0, kb * kElems, bar);
                        tc_load<CG>(b + 8192, &k.tb, n0 + 64, kb * kElems, bar);
                    } else {
                        tc_load<CG>(b, &k.tb, kb * kElems, n0, bar);
                    }
                    if (++stage == kTcStages) stage = 0, phase ^= 1;
                }
            }
            // Every stage is empty before this CTA leaves: the arrivals that say so reach both CTAs of a pair, in whatever order with those for the sums,
            // and must find the barriers of a CTA that is still there.  (After a wait that ran out the epilogue's, of 4 s, cover copies under way.)
            for (int i = 0; i < kTcStages && ok; ++i) {
                ok = tc_wait(empty + 8 * stage, phase ^ 1, k.err);
                if (++stage == kTcStages) stage = 0, phase ^= 1;
            }
        }
    } else if (warp == 1) {
        if (lane == 0 && rank == 0) {  // products
            constexpr uint32_t idesc = tc_idesc<CG, BN, kBits8, kArow, kBrow>();
            constexpr uint64_t astep = (kArow ? 2048 : 32) >> 4, bstep = (kBrow ? 2048 : 32) >> 4;
            uint32_t stage = 0, phase = 0, buf = 0, bphase = 0;
            bool ok = true;
            for (int u = first; u < k.units && ok; u += step) {
                const TcUnit t = tc_unit(k, u);
                if (!(ok = tc_wait(sums_empty + 8 * buf, bphase ^ 1, k.err))) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const int kb0 = t.split * k.kper, kb1 = min(k.kblocks, kb0 + k.kper);
                for (int kb = kb0; kb < kb1; ++kb) {
                    if (!(ok = tc_wait(full + 8 * stage, phase, k.err))) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint64_t a = tc_desc(base + stage * kTcStage, kArow), b = tc_desc(base + stage * kTcStage + kTcA, kBrow);
#pragma unroll
                    for (int i = 0; i < 4; ++i) tc_mma<CG, kBits8>(tmem + buf * BN, a + i * astep, b + i * bstep, idesc, kb > kb0 || i > 0);
                    tc_commit<CG>(empty + 8 * stage);
                    if (++stage == kTcStages) stage = 0, phase ^= 1;
                }
                if (!(k.drop && u == first)) tc_commit<CG>(sums_full + 8 * buf);
                buf ^= 1;
                if (buf == 0) bphase ^= 1;
            }
        }
    } else {  // sums: 32 rows, one in each lane, and half of the columns for each warp
        constexpr int COLS = BN / 2;
        const int quad = warp & 3, part = (warp - 2) >> 2;
        char* stage = smem_raw + (base - smem_u32(smem_raw)) + kTcStages * kTcStage + (warp - 2) * kTcEpiBytes;
        float* terms = reinterpret_cast<float*>(stage + 4096);  // of the warp's columns: factors, biases
        uint32_t buf = 0, bphase = 0;
        for (int u = first; u < k.units; u += step) {
            const TcUnit t = tc_unit(k, u);
            TcRows at;
            at.m0 = t.m * 128 * CG + (int)rank * 128 + quad * 32;
            at.n0 = t.n * BN + part * COLS;
            at.split = t.split;
            const int m = at.m0 + lane;
            at.on = m < k.M;
            at.at = (long long)m * k.N + at.n0;
            at.scale = k.e.row_scale && at.on ? k.e.row_scale[m] : 1.0f;
            __syncwarp();
#pragma unroll
            for (int j = lane; j < COLS; j += 32) {
                const bool in = at.n0 + j < k.N;
                terms[j] = in && k.e.col_scale ? k.e.col_scale[at.n0 + j] : 1.0f;
                terms[COLS + j] = in && k.e.bias ? k.e.bias[at.n0 + j] : 0.0f;
            }
            __syncwarp();
            // (one answer for the warp: a lane that gave up alone would leave the others in loads of the whole warp)
            if (!__all_sync(0xffffffffu, tc_wait(sums_full + 8 * buf, bphase, k.err, kTcSumsNs))) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t sums = tmem + buf * BN + part * COLS + ((uint32_t)(quad * 32) << 16);
            const bool whole = k.vec && k.splits == 1 && at.m0 < k.M;
            uint32_t r[32];
            tmem_load32(r, sums);
#pragma unroll 1
            for (int c = 0; c < COLS; c += 32) {
                const int n = at.n0 + c;
                const bool in = n < k.N && at.m0 < k.M;
                if (whole && k.e.residual && !(c & 32)) {
                    tc_rows<false>(k, const_cast<__nv_bfloat16*>(k.e.residual), at, n, stage);
                    __syncwarp();
                }
                float2 v[16];
                tmem_wait32(r);
                if (k.splits > 1) {
                    if (in) tc_part(k, at, c, r);
                } else {
                    tc_scale<COLS>(k, v, at, c, r, terms);
                }
                if (c + 32 < COLS) {
                    tmem_load32(r, sums + c + 32);
                } else {  // the buffer may be used again
                    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) {
                        if constexpr (CG == 2)
                            asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(in_first_cta(sums_empty + 8 * buf)) : "memory");
                        else
                            mbarrier_arrive(sums_empty + 8 * buf);
                    }
                }
                if (k.splits == 1 && in) tc_finish(k, at, c, v, stage);
                if (whole && (c & 32)) {
                    __syncwarp();
                    tc_rows<true>(k, k.e.out, at, n - 32, stage);
                    __syncwarp();
                }
            }
            buf ^= 1;
            if (buf == 0) bphase ^= 1;
        }
    }
    __syncwarp();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    if constexpr (CG == 2) cluster_barrier();
    else __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    if (warp == 1) {
        if constexpr (CG == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(kCols));
        else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(kCols));
    }
}

// The parts of a split contraction in order, and the epilogue.
template <int V> __global__ void __launch_bounds__(256) gemm_join_kernel(GemmEpilogue e, const float* partial, int splits, long long M, int N) {
    pdl_wait();
    pdl_launch_dependents();
    const long long item = (long long)blockIdx.x * 256 + threadIdx.x;
    const int per = (N + V - 1) / V;
    if (item >= M * per) return;
    const long long m = item / per;
    const int n = (int)(item - m * per) * V;
    const long long at = m * N + n;
    ColumnTerms<V> terms;
    terms.load(e, n);
    const Vec<__nv_bfloat16, V> residual = residual_at<V>(e, at);
    float v[V];
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = 0.0f;
#pragma unroll 4
    for (int s = 0; s < splits; ++s) {
        float p[V];
        load_vec<float, (V < 4 ? V : 4)>(*reinterpret_cast<float(*)[V < 4 ? V : 4]>(&p[0]), partial + (long long)s * M * N + at);
        if constexpr (V == 8) load_vec<float, 4>(*reinterpret_cast<float(*)[4]>(&p[4]), partial + (long long)s * M * N + at + 4);
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] += p[i];
    }
    finish<V>(e, v, terms, e.row_scale ? e.row_scale[m] : 1.0f, residual, at);
}

struct TcPlan {
    int cg, tiles_m, tiles_n, splits, kblocks, kper;
};
long long up(long long a, long long b) { return (a + b - 1) / b; }

// By estimated clocks: a stage of the contraction takes a pair 512 of them for 256 x 256 sums and one CTA 300 for 128 x 128, a tile 2000 to begin and end, a
// join 5000 and 8 bytes of traffic for each part's sum.  (128 x 2048 x 4096: 14.1 us so, by 32 CTAs in no parts 16.9; the bytes into an SM, 64 a clock, say 512 for
// 128 x 128 too, but with that the split cases came out slower: 18.4.)
TcPlan tc_plan(long long M, int N, long long K, bool bits8) {
    const int sms = device_sm_count();
    const long long kblocks = up(K, bits8 ? 128 : 64);
    TcPlan best{};
    double least = 0.0;
    for (int cg = 2; cg >= 1; --cg) {
        const long long tm = up(M, 128 * cg), tn = up(N, 128 * cg), slots = sms > cg ? sms / cg : 1;  // (without a device there is one SM)
        for (long long want = 1; want <= 64; ++want) {
            const long long kper = up(kblocks, want), splits = up(kblocks, kper);
            if (want > 1 && (kper < 4 || tm * tn * want > 2 * slots)) break;
            if (splits != want) continue;
            double t = (double)up(tm * tn * splits, slots) * (kper * (cg == 2 ? 512.0 : 300.0) + 2000.0);
            if (splits > 1) t += 5000.0 + (double)M * N * splits * 8.0 / 3500.0;
            if (best.cg == 0 || t < least) least = t, best = TcPlan{cg, (int)tm, (int)tn, (int)splits, (int)kblocks, (int)kper};
        }
    }
    return best;
}

PFN_cuTensorMapEncodeTiled_v12000 encoder() {
    static std::once_flag once;
    static PFN_cuTensorMapEncodeTiled_v12000 fn = nullptr;
    std::call_once(once, [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult q{};
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &q) == cudaSuccess && q == cudaDriverEntryPointSuccess)
            fn = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(f);
    });
    return fn;
}

// Boxes of 128 bytes: of the contraction and 128 rows, or of 64 rows and 64 steps of the contraction.
bool encode(CUtensorMap* m, const void* base, long long rows, long long K, long long r, long long c, bool bits8, bool* rows_dense) {
    const long long es = bits8 ? 1 : 2;
    if (reinterpret_cast<uintptr_t>(base) & 15) return false;
    *rows_dense = c != 1;
    if (*rows_dense && (bits8 || r != 1)) return false;
    const long long ld = *rows_dense ? c : r;
    if (ld <= 0 || ld * es % 16 || ld * es >= (1LL << 40)) return false;
    const PFN_cuTensorMapEncodeTiled_v12000 enc = encoder();
    if (!enc || refuse_tensor_maps()) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)(*rows_dense ? rows : K), (cuuint64_t)(*rows_dense ? K : rows)};
    const cuuint64_t strides[1] = {(cuuint64_t)(ld * es)};
    const cuuint32_t box[2] = {(cuuint32_t)(128 / es), *rows_dense ? 64u : 128u}, estr[2] = {1, 1};
    return enc(m, bits8 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, box, estr,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int CG> const void* tc_kernel(bool bits8, bool arow, bool brow) {
    constexpr int BN = 128 * CG;
    if (bits8) return (const void*)gemm_tc_kernel<CG, BN, true, false, false>;
    if (arow) return (const void*)gemm_tc_kernel<CG, BN, false, true, true>;
    return brow ? (const void*)gemm_tc_kernel<CG, BN, false, false, true> : (const void*)gemm_tc_kernel<CG, BN, false, false, false>;
}

}  // namespace

size_t gemm_partial_bytes(long long M, int N, long long K, bool bits8) {
    if (K == 0) return 0;
    const TcPlan p = tc_plan(M, N, K, bits8);
    return p.splits > 1 ? align_up((size_t)p.splits * M * N * 4, 256) : 0;
}

vmb_status launch_gemm_tc(const GemmProblem& p, bool bits8, float* partial, unsigned* err, cudaStream_t stream, bool* taken) {
    *taken = false;
    if (p.K < 1 || p.K > (1 << 30) || p.M > (1 << 30)) return VMB_OK;
    const TcPlan plan = tc_plan(p.M, p.N, p.K, bits8);
    if ((long long)plan.tiles_m * plan.tiles_n * plan.splits > (1 << 30)) return VMB_OK;
    TcKernel k;
    bool arow = false, brow = false;
    if (!encode(&k.ta, p.A, p.M, p.K, p.a_r, p.a_c, bits8, &arow) || !encode(&k.tb, p.B, p.N, p.K, p.b_r, p.b_c, bits8, &brow) || (arow && !brow)) return VMB_OK;
    k.e = p.e, k.partial = partial, k.err = err, k.M = p.M, k.N = p.N;
    k.tiles_m = plan.tiles_m, k.tiles_n = plan.tiles_n, k.splits = plan.splits, k.kblocks = plan.kblocks, k.kper = plan.kper;
    k.units = plan.tiles_m * plan.tiles_n * plan.splits;
    k.vec = epilogue_vectors(p);
    k.drop = drop_sums();
    const void* fn = plan.cg == 2 ? tc_kernel<2>(bits8, arow, brow) : tc_kernel<1>(bits8, arow, brow);
    if (cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, kTcSmem) != cudaSuccess) return VMB_ERR_CUDA;
    const int sms = device_sm_count(), slots = sms > plan.cg ? sms / plan.cg : 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)((k.units < slots ? k.units : slots) * plan.cg));
    cfg.blockDim = dim3(kTcThreads);
    cfg.dynamicSmemBytes = kTcSmem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = plan.cg, attr[1].val.clusterDim.y = 1, attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr, cfg.numAttrs = plan.cg == 2 ? 2 : 1;
    void* args[] = {&k};
    *taken = true;
    if (cudaLaunchKernelExC(&cfg, fn, args) != cudaSuccess) return VMB_ERR_CUDA;
    if (plan.splits == 1) return VMB_OK;
    GemmEpilogue e = p.e;
    const float* parts = partial;
    int splits = plan.splits, N = p.N;
    long long M = p.M;
    void* jargs[] = {&e, &parts, &splits, &M, &N};
    const long long items = M * (k.vec ? up(N, 8) : N);
    const void* join = k.vec ? (const void*)gemm_join_kernel<8> : (const void*)gemm_join_kernel<1>;
    return launch_kernel(join, dim3((unsigned)up(items, 256)), dim3(256), 0, jargs, stream) == cudaSuccess ? VMB_OK : VMB_ERR_CUDA;
}

}  // namespace vmb

extern "C" int vmb_testing_linear_plan(long long M, int N, long long K, int bits8, int* out) {
    const vmb::TcPlan p = vmb::tc_plan(M, N, K, bits8 != 0);
    out[0] = p.cg, out[1] = p.splits;
    return 0;
}
