// vmb_abi_layer.cu - the extern "C" entry points of the operators of a layer around the scan over tokens (declared in
// include/vmb.h): argument checks, workspace sizes, launches on the caller's stream.
#include <limits.h>

#include <initializer_list>

#include "layer_internal.h"
#include "vmb_internal.h"

namespace vmb {

namespace {

// The product of sizes, none negative; false where its bytes (up to 8 each) leave int64.
bool count(long long* out, std::initializer_list<long long> dims) {
    long long v = 1;
    for (long long d : dims) {
        if (d < 0 || (d != 0 && v > LLONG_MAX / 8 / d)) return false;
        v *= d;
    }
    *out = v;
    return true;
}
bool aligned(std::initializer_list<const void*> ps, size_t a) {
    for (const void* p : ps)
        if (reinterpret_cast<uintptr_t>(p) % a) return false;
    return true;
}
size_t esize(vmb_dtype dt) { return dt == VMB_BF16 ? 2 : 4; }
bool dtype_ok(vmb_dtype dt) { return dt == VMB_F32 || dt == VMB_BF16; }
bool act_ok(vmb_act a) { return a == VMB_ACT_NONE || a == VMB_ACT_SILU || a == VMB_ACT_GELU; }

vmb_status check_workspace(const void* ws) {
    if (!ws) return VMB_ERR_WORKSPACE;
    return aligned({ws}, 256) ? VMB_OK : VMB_ERR_MISALIGNED;
}

// Tokens of B sequences and what a launch over them needs; packed ones have T = total, the longest that there can be.
vmb_status token_sizes(int B, int* T, int64_t total, bool packed, int C, int W, vmb_dtype dt) {
    long long n;
    if (!dtype_ok(dt) || B < 0 || C < 0 || W < 0 || total < 0 || (!packed && *T < 0)) return VMB_ERR_INVALID_ARG;
    if (!packed && (!count(&n, {B, *T}) || n != total)) return VMB_ERR_INVALID_ARG;
    if (!count(&n, {total, C > W ? C : W}) || !count(&n, {B, W, C})) return VMB_ERR_INVALID_ARG;
    if (total > INT_MAX / 2 || B > (1 << 24) || C > (1 << 22)) return VMB_ERR_UNSUPPORTED;  // (rows and grids in 32 bits)
    if (packed) *T = (int)total;
    return VMB_OK;
}

// Batch and token strides of the i-th tensor: of `strides`, or dense.
bool take_strides(const int64_t* strides, int i, long long width, int T, bool packed, long long* b, long long* t) {
    *t = width, *b = width * T;
    if (!strides) return true;
    if (strides[2 * i] < 0 || strides[2 * i + 1] < 0) return false;
    *t = strides[2 * i + 1];
    if (!packed) *b = strides[2 * i];
    return true;
}

// What an empty problem leaves of its gradients: sums of nothing.  Outputs may be null.
struct Cleared {
    void* p;
    size_t bytes;
};
vmb_status clear(std::initializer_list<Cleared> outs, cudaStream_t stream) {
    for (const Cleared& o : outs)
        if (o.p && o.bytes && cudaMemsetAsync(o.p, 0, o.bytes, stream) != cudaSuccess) return VMB_ERR_CUDA;
    return VMB_OK;
}

// ------------------------------------------------------------ convolution

vmb_status conv_sizes(int B, int* T, int64_t total, bool packed, int C, int W, vmb_act act, vmb_dtype dt, bool* empty) {
    const vmb_status s = token_sizes(B, T, total, packed, C, W, dt);
    if (s != VMB_OK) return s;
    if (W < 1 || (act != VMB_ACT_NONE && act != VMB_ACT_SILU)) return VMB_ERR_INVALID_ARG;
    if (W > 4) return VMB_ERR_UNSUPPORTED;
    *empty = C == 0 || (B == 0 && total == 0);
    return VMB_OK;
}

// ------------------------------------------------------------ scan

vmb_status scan_sizes(int B, int* T, int64_t total, bool packed, int D, int N, vmb_dtype dt, bool* empty) {
    const vmb_status s = token_sizes(B, T, total, packed, D, N, dt);
    if (s != VMB_OK) return s;
    if (N < 1 && D > 0) return VMB_ERR_INVALID_ARG;
    if (N > 16) return VMB_ERR_UNSUPPORTED;
    *empty = D == 0 || (B == 0 && total == 0);
    // (segments, at least a chunk long, of all tiles of channels are counted in 32 bits, and so are partial sums' bytes in 64)
    long long n;
    const long long slots = scan_slots(B, *T, total, packed, kScanSaved) + 64, tiles = ((long long)D + 31) / 32;
    if (!count(&n, {slots, tiles}) || n > INT_MAX || !count(&n, {slots, D, 18}) || !count(&n, {tiles, total, 32})) return VMB_ERR_UNSUPPORTED;
    return VMB_OK;
}

vmb_status scan_args(TokenScanArgs& a, const void* x, const void* delta, const float* A, const void* Bm, const void* Cm, const float* Dskip,
                     const float* delta_bias, const void* z, const int64_t* strides, bool packed) {
    if (!A || (a.total > 0 && (!x || !delta || !Bm || !Cm))) return VMB_ERR_INVALID_ARG;
    if (!aligned({x, delta, Bm, Cm, z}, esize(a.dtype)) || !aligned({A, Dskip, delta_bias}, 4)) return VMB_ERR_MISALIGNED;
    a.x = x, a.delta = delta, a.A = A, a.Bm = Bm, a.Cm = Cm, a.skip = Dskip, a.bias = delta_bias, a.z = z;
    if (!take_strides(strides, 0, a.D, a.T, packed, &a.x_b, &a.x_t) || !take_strides(strides, 1, a.D, a.T, packed, &a.d_b, &a.d_t) ||
        !take_strides(strides, 2, a.N, a.T, packed, &a.B_b, &a.B_t) || !take_strides(strides, 3, a.N, a.T, packed, &a.C_b, &a.C_t) ||
        !take_strides(strides, 4, a.D, a.T, packed, &a.z_b, &a.z_t))
        return VMB_ERR_INVALID_ARG;
    // (places within a stage of 64 tokens are counted in 32 bits; a stride between tokens that there are not has no meaning)
    for (long long* t : {&a.x_t, &a.d_t, &a.B_t, &a.C_t, &a.z_t}) {
        if (a.total <= 1 || (!packed && a.T == 1)) *t = 0;
        if (*t >= (1 << 24)) return VMB_ERR_UNSUPPORTED;
    }
    return VMB_OK;
}

// ------------------------------------------------------------ norm and product

vmb_status rms_sizes(int64_t rows, int C, vmb_dtype dt, bool* empty) {
    long long n;
    if (!dtype_ok(dt) || rows < 0 || C < 0 || !count(&n, {rows, C})) return VMB_ERR_INVALID_ARG;
    *empty = n == 0;
    if (C > 8192 || rows > INT_MAX) return VMB_ERR_UNSUPPORTED;
    return VMB_OK;
}

vmb_status linear_sizes(int64_t M, int K, int N, bool* empty) {
    long long n;
    if (M < 0 || K < 0 || N < 0 || !count(&n, {M, K > N ? K : N}) || !count(&n, {K, N})) return VMB_ERR_INVALID_ARG;
    *empty = M == 0 || N == 0;
    if (M > (1 << 30) || K > (1 << 24) || N > (1 << 24)) return VMB_ERR_UNSUPPORTED;
    return VMB_OK;
}

}  // namespace

}  // namespace vmb

using namespace vmb;

extern "C" {

size_t vmb_causal_conv_workspace_bytes(int B, int T, int64_t total, int packed, int C, int W, vmb_dtype dtype) {
    bool empty = false;
    if (conv_sizes(B, &T, total, packed != 0, C, W, VMB_ACT_NONE, dtype, &empty) != VMB_OK) return 0;
    return empty ? 256 : conv_workspace_bytes(B, T, total, packed != 0, C, W, dtype);
}

vmb_status vmb_causal_conv_fwd(const void* x, const float* weight, const float* bias, const int64_t* strides, const void* initial_state,
                               const int32_t* offsets, void* y, void* final_state, int B, int T, int64_t total, int C, int W, vmb_act act,
                               vmb_dtype dtype, cudaStream_t stream) {
    bool empty = false;
    const vmb_status s = conv_sizes(B, &T, total, offsets != nullptr, C, W, act, dtype, &empty);
    if (s != VMB_OK || empty) return s;
    if (!weight || (total > 0 && (!x || !y || x == y))) return VMB_ERR_INVALID_ARG;
    if (final_state && (final_state == initial_state || final_state == x)) return VMB_ERR_INVALID_ARG;
    if (!aligned({x, y, initial_state, final_state}, esize(dtype)) || !aligned({weight, bias, offsets}, 4)) return VMB_ERR_MISALIGNED;
    ConvArgs a{x, weight, bias, W > 1 ? initial_state : nullptr, offsets, y, W > 1 ? final_state : nullptr, B, T, total, C, W, 0, 0, act, dtype};
    if (!take_strides(strides, 0, C, T, offsets != nullptr, &a.x_b, &a.x_t)) return VMB_ERR_INVALID_ARG;
    return launch_conv_fwd(a, stream);
}

vmb_status vmb_causal_conv_bwd(const void* x, const float* weight, const float* bias, const int64_t* strides, const void* initial_state,
                               const int32_t* offsets, const void* dy, const void* dfinal_state, void* dx, float* dweight, float* dbias,
                               void* dinitial_state, int B, int T, int64_t total, int C, int W, vmb_act act, vmb_dtype dtype, void* workspace,
                               size_t workspace_bytes, cudaStream_t stream) {
    bool empty = false;
    vmb_status s = conv_sizes(B, &T, total, offsets != nullptr, C, W, act, dtype, &empty);
    if (s != VMB_OK) return s;
    if (empty) return clear({{dweight, (size_t)C * W * 4}, {dbias, (size_t)C * 4}}, stream);
    if (!weight || !dweight || (total > 0 && (!x || !dy || !dx || dx == x || dx == dy))) return VMB_ERR_INVALID_ARG;
    if (dinitial_state && (dinitial_state == dfinal_state || dinitial_state == initial_state)) return VMB_ERR_INVALID_ARG;
    if (!aligned({x, dy, dx, initial_state, dfinal_state, dinitial_state}, esize(dtype)) || !aligned({weight, bias, dweight, dbias, offsets}, 4))
        return VMB_ERR_MISALIGNED;
    if ((s = check_workspace(workspace)) != VMB_OK) return s;
    ConvArgs a{x, weight, bias, W > 1 ? initial_state : nullptr, offsets, nullptr, nullptr, B, T, total, C, W, 0, 0, act, dtype};
    if (!take_strides(strides, 0, C, T, offsets != nullptr, &a.x_b, &a.x_t)) return VMB_ERR_INVALID_ARG;
    if (total <= 1 || (!offsets && T == 1)) a.x_t = 0;  // (no two tokens)
    if (a.x_t >= (1 << 24)) return VMB_ERR_UNSUPPORTED;
    a.dy = dy, a.dfinal = W > 1 ? dfinal_state : nullptr, a.dx = dx, a.dweight = dweight, a.dbias = dbias;
    a.dinitial = W > 1 ? dinitial_state : nullptr, a.ws = workspace, a.ws_bytes = workspace_bytes;
    return launch_conv_bwd(a, stream);
}

vmb_status vmb_causal_conv_step(const void* x, const float* weight, const float* bias, const int64_t* strides, void* state, const int32_t* slots,
                                void* y, int B, int T, int C, int W, int pool, vmb_act act, vmb_dtype dtype, cudaStream_t stream) {
    bool empty = false;
    long long total, n;
    if (pool < 0 || !count(&total, {B, T})) return VMB_ERR_INVALID_ARG;
    const vmb_status s = conv_sizes(B, &T, total, false, C, W, act, dtype, &empty);
    if (s != VMB_OK || empty || total == 0) return s;
    if (!count(&n, {pool, W, C}) || (!slots && pool < B)) return VMB_ERR_INVALID_ARG;
    if (!x || !weight || !y || x == y || (W > 1 && (!state || state == x || state == y))) return VMB_ERR_INVALID_ARG;
    if (!aligned({x, y, state}, esize(dtype)) || !aligned({weight, bias, slots}, 4)) return VMB_ERR_MISALIGNED;
    ConvArgs a{x, weight, bias, nullptr, nullptr, y, nullptr, B, T, total, C, W, 0, 0, act, dtype};
    if (!take_strides(strides, 0, C, T, false, &a.x_b, &a.x_t)) return VMB_ERR_INVALID_ARG;
    a.state = state, a.slots = slots, a.pool = pool;
    return launch_conv_step(a, stream);
}

size_t vmb_token_scan_workspace_bytes(int B, int T, int64_t total, int packed, int D, int N, int grads, vmb_dtype dtype) {
    bool empty = false;
    if (scan_sizes(B, &T, total, packed != 0, D, N, dtype, &empty) != VMB_OK) return 0;
    return empty ? 256 : token_scan_workspace_bytes(B, T, total, packed != 0, D, N, grads != 0, dtype);
}

size_t vmb_token_scan_saved_bytes(int B, int T, int64_t total, int packed, int D, int N) {
    bool empty = false;
    if (scan_sizes(B, &T, total, packed != 0, D, N, VMB_F32, &empty) != VMB_OK) return 0;
    return empty ? 256 : (size_t)scan_slots(B, T, total, packed != 0, kScanSaved) * D * N * 4 + 256;
}

vmb_status vmb_token_scan_fwd(const void* x, const void* delta, const float* A, const void* Bm, const void* Cm, const float* Dskip,
                              const float* delta_bias, const void* z, const int64_t* strides, const float* initial_state, const int32_t* offsets,
                              void* y, float* final_state, void* saved, int B, int T, int64_t total, int D, int N, unsigned flags, vmb_dtype dtype,
                              void* workspace, size_t workspace_bytes, cudaStream_t stream) {
    bool empty = false;
    const bool packed = offsets != nullptr;
    vmb_status s = scan_sizes(B, &T, total, packed, D, N, dtype, &empty);
    if (s != VMB_OK || (flags & ~VMB_FLAG_SOFTPLUS)) return s != VMB_OK ? s : VMB_ERR_INVALID_ARG;
    if (empty) return VMB_OK;
    TokenScanArgs a{};
    a.B = B, a.T = T, a.total = total, a.D = D, a.N = N, a.dtype = dtype, a.softplus = (flags & VMB_FLAG_SOFTPLUS) != 0;
    if ((s = scan_args(a, x, delta, A, Bm, Cm, Dskip, delta_bias, z, strides, packed)) != VMB_OK) return s;
    if (total > 0 && (!y || y == x || y == delta || y == Bm || y == Cm || y == z)) return VMB_ERR_INVALID_ARG;
    if (final_state && (const float*)final_state == initial_state) return VMB_ERR_INVALID_ARG;
    if (!aligned({y}, esize(dtype)) || !aligned({initial_state, final_state, offsets}, 4) || !aligned({saved}, 16)) return VMB_ERR_MISALIGNED;
    if ((s = check_workspace(workspace)) != VMB_OK) return s;
    a.initial = initial_state, a.offsets = offsets, a.y = y, a.final = final_state, a.saved = (float*)saved;
    a.ws = workspace, a.ws_bytes = workspace_bytes;
    return launch_token_scan_fwd(a, stream);
}

vmb_status vmb_token_scan_bwd(const void* x, const void* delta, const float* A, const void* Bm, const void* Cm, const float* Dskip,
                              const float* delta_bias, const void* z, const int64_t* strides, const int32_t* offsets, const void* dy,
                              const float* dfinal_state, const void* saved, void* dx, void* ddelta, float* dA, void* dBm, void* dCm, float* dDskip,
                              float* ddelta_bias, void* dz, float* dinitial_state, int B, int T, int64_t total, int D, int N, unsigned flags,
                              vmb_dtype dtype, void* workspace, size_t workspace_bytes, cudaStream_t stream) {
    bool empty = false;
    const bool packed = offsets != nullptr;
    vmb_status s = scan_sizes(B, &T, total, packed, D, N, dtype, &empty);
    if (s != VMB_OK || (flags & ~VMB_FLAG_SOFTPLUS)) return s != VMB_OK ? s : VMB_ERR_INVALID_ARG;
    if (empty)  // (without channels B's and C's gradients have elements still)
        return clear({{dA, (size_t)D * N * 4}, {dDskip, (size_t)D * 4}, {ddelta_bias, (size_t)D * 4}, {dBm, (size_t)total * N * esize(dtype)},
                      {dCm, (size_t)total * N * esize(dtype)}}, stream);
    TokenScanArgs a{};
    a.B = B, a.T = T, a.total = total, a.D = D, a.N = N, a.dtype = dtype, a.softplus = (flags & VMB_FLAG_SOFTPLUS) != 0;
    if ((s = scan_args(a, x, delta, A, Bm, Cm, Dskip, delta_bias, z, strides, packed)) != VMB_OK) return s;
    if (!dA || (total > 0 && (!dy || !saved || !dx || !ddelta || !dBm || !dCm || (z && !dz)))) return VMB_ERR_INVALID_ARG;
    if (dinitial_state && (const float*)dinitial_state == dfinal_state) return VMB_ERR_INVALID_ARG;
    for (const void* out : {dx, ddelta, dBm, dCm, dz})
        if (out && (out == x || out == delta || out == Bm || out == Cm || out == z || out == dy)) return VMB_ERR_INVALID_ARG;
    if (!aligned({dy, dx, ddelta, dBm, dCm, dz}, esize(dtype)) || !aligned({dA, dDskip, ddelta_bias, dinitial_state, dfinal_state, offsets}, 4) ||
        !aligned({saved}, 16))
        return VMB_ERR_MISALIGNED;
    if ((s = check_workspace(workspace)) != VMB_OK) return s;
    a.offsets = offsets, a.saved = (float*)const_cast<void*>(saved), a.dy = dy, a.dfinal = dfinal_state;
    a.dx = dx, a.ddelta = ddelta, a.dA = dA, a.dB = dBm, a.dC = dCm, a.dskip = dDskip, a.dbias = ddelta_bias, a.dz = z ? dz : nullptr;
    a.dinitial = dinitial_state, a.ws = workspace, a.ws_bytes = workspace_bytes;
    return launch_token_scan_bwd(a, stream);
}

vmb_status vmb_token_scan_step(const void* x, const void* delta, const float* A, const void* Bm, const void* Cm, const float* Dskip,
                               const float* delta_bias, const void* z, const int64_t* strides, float* state, const int32_t* slots, void* y, int B,
                               int T, int D, int N, int pool, unsigned flags, vmb_dtype dtype, cudaStream_t stream) {
    bool empty = false;
    long long total, n;
    if (pool < 0 || !count(&total, {B, T}) || (flags & ~VMB_FLAG_SOFTPLUS)) return VMB_ERR_INVALID_ARG;
    vmb_status s = scan_sizes(B, &T, total, false, D, N, dtype, &empty);
    if (s != VMB_OK || empty || total == 0) return s;
    if (!count(&n, {pool, D, N}) || (!slots && pool < B)) return VMB_ERR_INVALID_ARG;
    if (!count(&n, {B, ((long long)D + 31) / 32}) || n > INT_MAX) return VMB_ERR_UNSUPPORTED;
    TokenScanArgs a{};
    a.B = B, a.T = T, a.total = total, a.D = D, a.N = N, a.dtype = dtype, a.softplus = (flags & VMB_FLAG_SOFTPLUS) != 0;
    if ((s = scan_args(a, x, delta, A, Bm, Cm, Dskip, delta_bias, z, strides, false)) != VMB_OK) return s;
    if (!state || !y || y == x || y == delta || y == Bm || y == Cm || y == z) return VMB_ERR_INVALID_ARG;
    if (!aligned({y}, esize(dtype)) || !aligned({state, slots}, 4)) return VMB_ERR_MISALIGNED;
    a.y = y, a.state = state, a.slots = slots, a.pool = pool;
    return launch_token_scan_step(a, stream);
}

size_t vmb_rms_norm_workspace_bytes(int64_t rows, int C, vmb_dtype dtype) {
    bool empty = false;
    if (rms_sizes(rows, C, dtype, &empty) != VMB_OK) return 0;
    return empty ? 256 : rms_workspace_bytes(rows, C, dtype);
}

vmb_status vmb_rms_norm_fwd(const void* x, const void* residual, const float* weight, void* y, void* sum, float* scale, float* rstd, int64_t rows,
                            int C, float eps, vmb_dtype dtype, cudaStream_t stream) {
    bool empty = false;
    const vmb_status s = rms_sizes(rows, C, dtype, &empty);
    if (s != VMB_OK) return s;
    if (!(eps >= 0.0f)) return VMB_ERR_INVALID_ARG;
    if (rows > 0 && C == 0 && (scale || rstd)) return VMB_ERR_INVALID_ARG;  // (no channels have no mean)
    if (empty) return VMB_OK;
    if (!x || !y || x == y || y == residual || (residual && (!sum || sum == y || sum == x || sum == residual))) return VMB_ERR_INVALID_ARG;
    if (!aligned({x, residual, sum}, esize(dtype)) || (!scale && !aligned({y}, esize(dtype))) || !aligned({weight, scale, rstd}, 4))
        return VMB_ERR_MISALIGNED;
    RmsArgs a{x, residual, weight, y, residual ? sum : nullptr, scale, rstd, rows, C, eps, scale != nullptr, dtype};
    return launch_rms_fwd(a, stream);
}

vmb_status vmb_rms_norm_bwd(const void* x, const float* weight, const float* rstd, const void* dy, const void* dsum, void* dx, float* dweight,
                            int64_t rows, int C, vmb_dtype dtype, void* workspace, size_t workspace_bytes, cudaStream_t stream) {
    bool empty = false;
    vmb_status s = rms_sizes(rows, C, dtype, &empty);
    if (s != VMB_OK) return s;
    if (empty) return clear({{dweight, (size_t)C * 4}}, stream);
    if (!x || !rstd || !dy || !dx || dx == x || dx == dy || dx == dsum) return VMB_ERR_INVALID_ARG;
    if (!aligned({x, dy, dsum, dx}, esize(dtype)) || !aligned({weight, rstd, dweight}, 4)) return VMB_ERR_MISALIGNED;
    if ((s = check_workspace(workspace)) != VMB_OK) return s;
    RmsArgs a{x, nullptr, weight, nullptr, nullptr, nullptr, const_cast<float*>(rstd), rows, C, 0.0f, false, dtype};
    a.dy = dy, a.dsum = dsum, a.dx = dx, a.dweight = dweight, a.ws = workspace, a.ws_bytes = workspace_bytes;
    return launch_rms_bwd(a, stream);
}

size_t vmb_linear_workspace_bytes(int64_t M, int K, int N, int grads) {
    bool empty = false;
    if (linear_sizes(M, K, N, &empty) != VMB_OK) return 0;
    return empty ? 256 : linear_workspace_bytes(M, K, N, grads != 0);
}

vmb_status vmb_linear_fwd(const void* x, int64_t x_stride, const void* weight, const float* x_scale, const float* weight_scale, const float* bias,
                          const void* residual, void* y, void* pre, int64_t M, int K, int N, vmb_act act, void* workspace, size_t workspace_bytes,
                          cudaStream_t stream) {
    bool empty = false;
    vmb_status s = linear_sizes(M, K, N, &empty);
    if (s != VMB_OK) return s;
    if (!act_ok(act) || !x_scale != !weight_scale || x_stride < 0) return VMB_ERR_INVALID_ARG;
    if (empty) return VMB_OK;
    if (!y || (K > 0 && (!x || !weight)) || y == x || y == weight || y == residual || y == pre || (pre && (pre == x || pre == weight || pre == residual)))
        return VMB_ERR_INVALID_ARG;
    long long n;
    if (!count(&n, {M, x_stride})) return VMB_ERR_INVALID_ARG;
    if ((!x_scale && !aligned({x, weight}, 2)) || !aligned({residual, y, pre}, 2) || !aligned({x_scale, weight_scale, bias}, 4)) return VMB_ERR_MISALIGNED;
    if ((s = check_workspace(workspace)) != VMB_OK) return s;
    LinearArgs a{x, weight, x_scale, weight_scale, bias, residual, y, pre, M, K, N, x_stride, act};
    a.ws = workspace, a.ws_bytes = workspace_bytes;
    return launch_linear_fwd(a, stream);
}

vmb_status vmb_linear_bwd(const void* x, int64_t x_stride, const void* weight, const void* pre, const void* dy, void* dx, void* dweight, float* dbias,
                          int64_t M, int K, int N, vmb_act act, void* workspace, size_t workspace_bytes, cudaStream_t stream) {
    bool empty = false;
    vmb_status s = linear_sizes(M, K, N, &empty);
    if (s != VMB_OK) return s;
    if (!act_ok(act) || x_stride < 0) return VMB_ERR_INVALID_ARG;
    if (empty) return clear({{dx, (size_t)M * K * 2}, {dweight, (size_t)N * K * 2}, {dbias, (size_t)N * 4}}, stream);
    if (!dy || (act != VMB_ACT_NONE && !pre) || (K > 0 && ((dx && !weight) || (dweight && !x)))) return VMB_ERR_INVALID_ARG;
    for (const void* out : {dx, dweight})
        if (out && (out == x || out == weight || out == pre || out == dy)) return VMB_ERR_INVALID_ARG;
    if (dx && dx == dweight) return VMB_ERR_INVALID_ARG;
    long long n;
    if (!count(&n, {M, x_stride})) return VMB_ERR_INVALID_ARG;
    if (!aligned({x, weight, pre, dy, dx, dweight}, 2) || !aligned({dbias}, 4)) return VMB_ERR_MISALIGNED;
    if ((s = check_workspace(workspace)) != VMB_OK) return s;
    LinearArgs a{x, weight, nullptr, nullptr, nullptr, nullptr, nullptr, const_cast<void*>(pre), M, K, N, x_stride, act};
    a.dy = dy, a.dx = dx, a.dweight = dweight, a.dbias = dbias, a.ws = workspace, a.ws_bytes = workspace_bytes;
    return launch_linear_bwd(a, stream);
}

}  // extern "C"
