// token_scan.cuh - what the forward and the gradients of the selective scan over tokens share: where a segment of a
// sequence lies, the states of a lane, the sums over the lanes of a channel, and the staging of tokens in shared memory (adjoint).
//
// Channels lie side by side in a token's row, and a CTA takes 64 of them, a tile.  The states of a channel lie in the lanes of a group, two in the
// forward and four elsewhere; a lane prepares one token of every two or four (its step size, its product with x, its gate) and
// hands them to the others by shuffles.
#pragma once

#include "layer_common.cuh"
#include "layer_internal.h"
#include "vmb_internal.h"

namespace vmb {

constexpr int kScanCh = 64, kScanThreads = 256;  // channels of a tile; threads of the adjoint's CTAs

struct ScanKernel {
    TokenScanArgs a;
    int seg;          // tokens of a segment, a multiple of kScanChunk
    int segs_per;     // segments of a sequence (dense)
    int slots;        // places of segments; packed: the segments of sequence b start at offsets[b] / seg + b
    int tiles;        // of channels
    bool vec, pair;   // rows allow copies of 16 bytes, and of two channels
    float* local;     // [slots][D][NP]: what a segment gives from a zero state (gradients: to the state before it)
    float* decay;     // [slots][D]: the sum of a segment's step sizes
    float* bc;        // gradients: [tiles][total][32]
    float* params;    // gradients: [slots][D N | D | D]
};

inline int padded_states(int N) { return N <= 4 ? 4 : N <= 8 ? 8 : 16; }
// Fills what follows from the sizes and a segment's length.
void token_scan_plan(ScanKernel& k, int seg);
size_t token_scan_forward_bytes(int B, int T, long long total, bool packed, int D, int N);
constexpr int kClearBlocks = 8;  // blocks for each tile that clear the rows of no sequence

struct ScanSegment {
    int b, s, segs;
    long long first;  // its first row of all
    int len;          // its tokens
    long long seq_len;
    long long place;  // of the sequence's first segment, and of its first chunk
    long long chunk;
    bool live;        // false: nothing lies here
};

// Called by whole warps.
__device__ __forceinline__ ScanSegment scan_segment(const ScanKernel& k, long long slot) {
    const TokenScanArgs& a = k.a;
    ScanSegment g;
    if (a.offsets) {
        const auto start = [&](int b) {
            const long long o = a.offsets[b];
            return o < 0 ? 0 : o > a.total ? a.total : o;
        };
        g.b = last_at_most(a.B, slot, [&](int b) { return start(b) / k.seg + b; });
        g.live = false;
        if (g.b < 0 || g.b >= a.B) return g;
        long long s0, e0;
        sequence_span(a.offsets, g.b, a.total, &s0, &e0);
        g.place = s0 / k.seg + g.b;
        g.chunk = s0 / kScanSaved + g.b;
        g.s = (int)(slot - g.place);
        g.seq_len = e0 - s0;
        g.first = s0;
    } else {
        g.b = (int)(slot / k.segs_per);
        g.s = (int)(slot - (long long)g.b * k.segs_per);
        g.place = (long long)g.b * k.segs_per;
        g.chunk = (long long)g.b * ((a.T + kScanSaved - 1) / kScanSaved);
        g.seq_len = a.T;
        g.first = (long long)g.b * a.T;
    }
    g.segs = (int)((g.seq_len + k.seg - 1) / k.seg);
    if (g.segs < 1) g.segs = 1;  // (an empty sequence still hands on its state)
    g.live = g.s >= 0 && g.s < g.segs;
    const long long off = (long long)g.s * k.seg;
    g.first += off;
    g.len = (int)(g.seq_len - off < k.seg ? g.seq_len - off : k.seg);
    return g;
}

// Packed sequences: reports offsets that decrease or leave the tokens; `blocks` blocks of a launch share them out (a segment does not see all of
// them: where they decrease, a place may belong to two sequences).
__device__ __forceinline__ void check_offsets(const TokenScanArgs& a, long long block, long long blocks) {
    bool bad = false;
    for (long long i = block * blockDim.x + threadIdx.x; i <= a.B; i += blocks * blockDim.x) {
        const int o = a.offsets[i];
        bad |= o < 0 || o > a.total || (i > 0 && o < a.offsets[i - 1]);
    }
    if (bad) atomicOr(&((WsHeader*)a.ws)->err, kErrBounds);
}

// The first element of a tensor's row `first` in a segment (batch rows may be strided in dense inputs).
template <typename T>
__device__ __forceinline__ const T* scan_row(const void* p, const TokenScanArgs& a, const ScanSegment& g, long long bs, long long ts) {
    if (a.offsets) return (const T*)p + g.first * ts;
    return (const T*)p + g.b * bs + (g.first - (long long)g.b * a.T) * ts;
}

// Pitch of a staged token's row: 16 (bf16) or 32 (fp32) bytes behind the channels keep the four tokens that a warp reads at once in
// different banks.
template <typename T> constexpr int scan_pitch() { return kScanCh * (int)sizeof(T) + (sizeof(T) == 2 ? 16 : 32); }

// Copies `tokens` rows of 64 channels from src (row stride ts, `cols` channels there) to shared memory; rows from `len` on and
// channels from `cols` on are zeros.
template <typename T>
__device__ __forceinline__ void stage_rows(char* dst, const T* src, long long ts, int tokens, int len, int cols, bool vec) {
    constexpr int V = 16 / (int)sizeof(T), per = kScanCh / V;
    if (vec) {
        for (int i = threadIdx.x; i < tokens * per; i += kScanThreads) {
            const int t = i / per, c = (i % per) * V;
            const bool in = t < len && c < cols;
            cp_async16(dst + t * scan_pitch<T>() + c * (int)sizeof(T), in ? (const void*)(src + t * ts + c) : (const void*)src, in ? 16 : 0);
        }
    } else {
        for (int i = threadIdx.x; i < tokens * kScanCh; i += kScanThreads) {
            const int t = i / kScanCh, c = i % kScanCh;
            *reinterpret_cast<T*>(dst + t * scan_pitch<T>() + c * (int)sizeof(T)) = t < len && c < cols ? src[t * ts + c] : io<T>::to(0.0f);
        }
    }
}
template <typename T> __device__ __forceinline__ float staged(const char* p, int t, int c) {
    return io<T>::ld(reinterpret_cast<const T*>(p + t * scan_pitch<T>()) + c);
}
// C of TOK rows in fp32, NP values each (N of them read, zeros behind and from row len on).
template <typename T, int NP, int TOK> __device__ __forceinline__ void stage_states(float* dst, const T* C, long long C_t, int N, int len) {
    constexpr int kEach = (TOK * NP + kScanThreads - 1) / kScanThreads;
    float v[kEach];
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        const int i = threadIdx.x + j * kScanThreads, t = i / NP, n = i % NP;
        v[j] = t < TOK && t < len && n < N ? io<T>::ld(C + t * C_t + n) : 0.0f;
    }
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        const int i = threadIdx.x + j * kScanThreads;
        if (i < TOK * NP) dst[i] = v[j];
    }
}

// A lane's states, in pairs: SPL = NP / 4 of them (one state alone is paired with a zero).
template <int SPL> struct Pairs {
    static constexpr int P = (SPL + 1) / 2;
    float2 v[P];
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int p = 0; p < P; ++p) v[p] = make_float2(0.0f, 0.0f);
    }
    // from shared memory or a padded row of global memory
    __device__ __forceinline__ void load(const float* s) {
        if constexpr (SPL >= 4) {
#pragma unroll
            for (int i = 0; i < SPL / 4; ++i) {
                const float4 x = reinterpret_cast<const float4*>(s)[i];
                v[2 * i] = make_float2(x.x, x.y), v[2 * i + 1] = make_float2(x.z, x.w);
            }
        } else if constexpr (SPL == 2) {
            v[0] = *reinterpret_cast<const float2*>(s);
        } else {
            v[0] = make_float2(s[0], 0.0f);
        }
    }
    __device__ __forceinline__ void store(float* s) const {
        if constexpr (SPL >= 4) {
#pragma unroll
            for (int i = 0; i < SPL / 4; ++i) reinterpret_cast<float4*>(s)[i] = make_float4(v[2 * i].x, v[2 * i].y, v[2 * i + 1].x, v[2 * i + 1].y);
        } else if constexpr (SPL == 2) *reinterpret_cast<float2*>(s) = v[0];
        else s[0] = v[0].x;
    }
    // from and to a row of N values at its n0-th
    __device__ __forceinline__ void load_some(const float* s, int n0, int N) {
#pragma unroll
        for (int p = 0; p < P; ++p)
            v[p] = make_float2(n0 + 2 * p < N ? s[2 * p] : 0.0f, SPL > 1 && n0 + 2 * p + 1 < N ? s[2 * p + 1] : 0.0f);
    }
    __device__ __forceinline__ void store_some(float* s, int n0, int N) const {
#pragma unroll
        for (int p = 0; p < P; ++p) {
            if (n0 + 2 * p < N) s[2 * p] = v[p].x;
            if (SPL > 1 && n0 + 2 * p + 1 < N) s[2 * p + 1] = v[p].y;
        }
    }
};
__device__ __forceinline__ float2 twice(float v) { return make_float2(v, v); }

// 2^(A log2 e  dt) of a lane's states
template <int SPL> __device__ __forceinline__ void decays(Pairs<SPL>& a, const Pairs<SPL>& A2, float dt) {
#pragma unroll
    for (int p = 0; p < Pairs<SPL>::P; ++p) {
        const float2 e = __fmul2_rn(A2.v[p], twice(dt));
        a.v[p] = make_float2(ex2(e.x), ex2(e.y));
    }
}

// The sums over the four lanes of a channel of four values: lane q gets that of v[q].
__device__ __forceinline__ float quad_sums(float v0, float v1, float v2, float v3) {
    const bool hi = threadIdx.x & 2, odd = threadIdx.x & 1;
    const float s0 = hi ? v0 : v2, s1 = hi ? v1 : v3;
    float k0 = hi ? v2 : v0, k1 = hi ? v3 : v1;
    k0 += __shfl_xor_sync(0xffffffffu, s0, 2);
    k1 += __shfl_xor_sync(0xffffffffu, s1, 2);
    return (odd ? k1 : k0) + __shfl_xor_sync(0xffffffffu, odd ? k0 : k1, 1);
}
__device__ __forceinline__ float from_lane(float v, int q) { return __shfl_sync(0xffffffffu, v, (threadIdx.x & 28) | q); }

}  // namespace vmb
