// vmb_abi_mixer.cu - the extern "C" entry points of the token mixer's operators (declared in
// include/vmb.h): argument checks, workspace sizes, launches on the caller's stream.
#include <limits.h>

#include <initializer_list>

#include "delta_internal.h"
#include "mixer_internal.h"
#include "vmb_internal.h"

namespace vmb {

namespace {

bool mul_ok(long long a, long long b, long long* out) {
    if (a < 0 || b < 0) return false;
    if (a != 0 && b > LLONG_MAX / a) return false;
    *out = a * b;
    return true;
}
// Bytes of up to 8 per element stay within int64.
bool count(long long* out, std::initializer_list<long long> dims) {
    long long v = 1, bytes;
    for (long long d : dims)
        if (!mul_ok(v, d, &v)) return false;
    *out = v;
    return mul_ok(v, 8, &bytes);
}
bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
size_t esize(vmb_dtype dt) { return dt == VMB_BF16 ? 2 : 4; }
bool dtype_ok(vmb_dtype dt) { return dt == VMB_F32 || dt == VMB_BF16; }

// The longest sequence: of packed ones T is a bound, and none is longer than all tokens.
int longest(int T, int64_t total, bool packed) { return packed && total >= 0 && T > total ? (int)total : T; }

// Sizes shared by the delta rule's calls; *empty: no tokens and no states.
vmb_status delta_sizes(int B, int T, int64_t total, bool packed, int Hk, int Hv, int Dk, int Dv, vmb_dtype dt, bool* empty) {
    if (!dtype_ok(dt) || B < 0 || T < 0 || total < 0 || Hk < 0 || Hv < 0 || Dk < 0 || Dv < 0) return VMB_ERR_INVALID_ARG;
    long long n;
    if (!packed) {
        if (!mul_ok(B, T, &n) || n != total) return VMB_ERR_INVALID_ARG;
    }
    if (!count(&n, {total, Hv, Dk > Dv ? Dk : Dv}) || !count(&n, {B, Hv, Dk, Dv})) return VMB_ERR_INVALID_ARG;
    *empty = n == 0 || Hk == 0;
    if (*empty) return VMB_OK;
    if (Hv % Hk) return VMB_ERR_INVALID_ARG;
    if (Dk > 128) return VMB_ERR_UNSUPPORTED;
    const long long chunks = ((long long)T + 63) / 64, slices = ((long long)Dv + 63) / 64;
    // (grids, the places of chunk states and of workspace parts stay within 31 and 63 bits)
    if (!count(&n, {B, Hv, slices + 2}) || n > INT_MAX / 512) return VMB_ERR_UNSUPPORTED;
    if (!count(&n, {B, Hv, chunks}) || n > INT_MAX) return VMB_ERR_UNSUPPORTED;
    const long long slots = packed ? total / 64 + B : B * chunks;
    if (slots > INT_MAX) return VMB_ERR_UNSUPPORTED;
    if (!count(&n, {slots, Hv, Dk, Dv})) return VMB_ERR_INVALID_ARG;
    return VMB_OK;
}

vmb_status delta_strides(DeltaArgs& a, const int64_t* strides) {
    a.q_t = a.k_t = (long long)a.Hk * a.Dk;
    a.v_t = (long long)a.Hv * a.Dv;
    a.q_b = a.k_b = a.q_t * a.T;
    a.v_b = a.v_t * a.T;
    if (!strides) return VMB_OK;
    for (int i = 0; i < 6; ++i)
        if (strides[i] < 0) return VMB_ERR_INVALID_ARG;
    a.q_b = strides[0], a.q_t = strides[1], a.k_b = strides[2], a.k_t = strides[3], a.v_b = strides[4], a.v_t = strides[5];
    return VMB_OK;
}

vmb_status check_workspace(const void* ws) {
    if (!ws) return VMB_ERR_WORKSPACE;
    return aligned(ws, 256) ? VMB_OK : VMB_ERR_MISALIGNED;
}

size_t saved_residuals_off(const DeltaArgs& a) {
    return align_up((size_t)delta_slots(a.B, a.T, a.total, a.offsets != nullptr) * a.Hv * a.Dv * a.Dk * esize(a.dtype), 256);
}

// A dummy that says "packed" in size queries.
const int kPacked = 0;

}  // namespace

}  // namespace vmb

using namespace vmb;

extern "C" {

size_t vmb_delta_rule_workspace_bytes(int B, int T, int64_t total, int packed, int Hk, int Hv, int Dk, int Dv, int grads,
                                      vmb_dtype dtype) {
    bool empty = false;
    T = longest(T, total, packed != 0);
    if (delta_sizes(B, T, total, packed != 0, Hk, Hv, Dk, Dv, dtype, &empty) != VMB_OK) return 0;
    if (empty) return 256;
    DeltaArgs a;
    a.offsets = packed ? &kPacked : nullptr;
    a.B = B, a.T = T, a.total = total, a.Hk = Hk, a.Hv = Hv, a.Dk = Dk, a.Dv = Dv, a.dtype = dtype;
    return plan_delta(a, grads != 0, device_sm_count()).bytes;
}

size_t vmb_delta_rule_saved_bytes(int B, int T, int64_t total, int packed, int Hv, int Dk, int Dv, vmb_dtype dtype) {
    bool empty = false;
    T = longest(T, total, packed != 0);
    if (delta_sizes(B, T, total, packed != 0, 1, Hv, Dk, Dv, dtype, &empty) != VMB_OK) return 0;
    if (empty) return 256;
    DeltaArgs a;
    a.offsets = packed ? &kPacked : nullptr;
    a.B = B, a.T = T, a.total = total, a.Hk = 1, a.Hv = Hv, a.Dk = Dk, a.Dv = Dv, a.dtype = dtype;
    return saved_residuals_off(a) + (size_t)total * Hv * Dv * esize(dtype);
}

vmb_status vmb_delta_rule_fwd(const void* q, const void* k, const void* v, const void* g, const void* beta, const int64_t* strides,
                              const float* initial_state, const int32_t* offsets, void* o, float* final_state, void* saved, int B,
                              int T, int64_t total, int Hk, int Hv, int Dk, int Dv, float scale, vmb_dtype dtype, void* workspace,
                              size_t workspace_bytes, cudaStream_t stream) {
    bool empty = false;
    T = longest(T, total, offsets != nullptr);
    vmb_status s = delta_sizes(B, T, total, offsets != nullptr, Hk, Hv, Dk, Dv, dtype, &empty);
    if (s != VMB_OK || empty) return s;
    const size_t es = esize(dtype);
    if (total > 0 && (!q || !k || !v || !g || !beta || !o)) return VMB_ERR_INVALID_ARG;
    if (final_state && (const float*)final_state == initial_state) return VMB_ERR_INVALID_ARG;
    if (o && (o == q || o == k || o == v)) return VMB_ERR_INVALID_ARG;
    if (!aligned(q, es) || !aligned(k, es) || !aligned(v, es) || !aligned(g, es) || !aligned(beta, es) || !aligned(o, es) ||
        !aligned(initial_state, 4) || !aligned(final_state, 4) || !aligned(offsets, 4) || !aligned(saved, 16))
        return VMB_ERR_MISALIGNED;
    if ((s = check_workspace(workspace)) != VMB_OK) return s;
    DeltaArgs a;
    a.q = q, a.k = k, a.v = v, a.g = g, a.beta = beta, a.initial = initial_state, a.offsets = offsets, a.o = o, a.final = final_state;
    a.B = B, a.T = T, a.total = total, a.Hk = Hk, a.Hv = Hv, a.Dk = Dk, a.Dv = Dv, a.scale = scale, a.dtype = dtype;
    a.ws = workspace, a.ws_bytes = workspace_bytes;
    if ((s = delta_strides(a, strides)) != VMB_OK) return s;
    if (saved) {
        a.saved = saved;
        a.saved_r = (char*)saved + saved_residuals_off(a);
    }
    return launch_delta_fwd(a, stream);
}

vmb_status vmb_delta_rule_bwd(const void* q, const void* k, const void* g, const void* beta, const int64_t* strides,
                              const int32_t* offsets, const void* dout, const float* dfinal_state, const void* saved, void* dq,
                              void* dk, void* dv, void* dg, void* dbeta, float* dinitial_state, int B, int T, int64_t total, int Hk,
                              int Hv, int Dk, int Dv, float scale, vmb_dtype dtype, void* workspace, size_t workspace_bytes,
                              cudaStream_t stream) {
    bool empty = false;
    T = longest(T, total, offsets != nullptr);
    vmb_status s = delta_sizes(B, T, total, offsets != nullptr, Hk, Hv, Dk, Dv, dtype, &empty);
    if (s != VMB_OK || empty) return s;
    const size_t es = esize(dtype);
    if (total > 0 && (!q || !k || !g || !beta || !dout || !saved || !dq || !dk || !dv || !dg || !dbeta)) return VMB_ERR_INVALID_ARG;
    if (dinitial_state && (const float*)dinitial_state == dfinal_state) return VMB_ERR_INVALID_ARG;
    if (!aligned(q, es) || !aligned(k, es) || !aligned(g, es) || !aligned(beta, es) || !aligned(dout, es) || !aligned(dq, es) ||
        !aligned(dk, es) || !aligned(dv, es) || !aligned(dg, es) || !aligned(dbeta, es) || !aligned(dfinal_state, 4) ||
        !aligned(dinitial_state, 4) || !aligned(offsets, 4) || !aligned(saved, 16))
        return VMB_ERR_MISALIGNED;
    if ((s = check_workspace(workspace)) != VMB_OK) return s;
    DeltaArgs a;
    a.q = q, a.k = k, a.g = g, a.beta = beta, a.offsets = offsets, a.dout = dout, a.dfinal = dfinal_state;
    a.dq = dq, a.dk = dk, a.dv = dv, a.dg = dg, a.dbeta = dbeta, a.dinitial = dinitial_state;
    a.B = B, a.T = T, a.total = total, a.Hk = Hk, a.Hv = Hv, a.Dk = Dk, a.Dv = Dv, a.scale = scale, a.dtype = dtype;
    a.ws = workspace, a.ws_bytes = workspace_bytes;
    if ((s = delta_strides(a, strides)) != VMB_OK) return s;
    a.saved = const_cast<void*>(saved);
    a.saved_r = (char*)a.saved + saved_residuals_off(a);
    return launch_delta_bwd(a, stream);
}

vmb_status vmb_delta_rule_step(const void* q, const void* k, const void* v, const void* g, const void* beta, const int64_t* strides,
                               float* state, const int32_t* slots, void* o, int B, int T, int Hk, int Hv, int Dk, int Dv, int pool,
                               float scale, vmb_dtype dtype, cudaStream_t stream) {
    bool empty = false;
    long long total = 0, n;
    if (B < 0 || T < 0 || pool < 0 || !mul_ok(B, T, &total)) return VMB_ERR_INVALID_ARG;
    vmb_status s = delta_sizes(B, T, total, false, Hk, Hv, Dk, Dv, dtype, &empty);
    if (s != VMB_OK || empty || T == 0) return s;
    if (!count(&n, {pool, Hv, Dk, Dv})) return VMB_ERR_INVALID_ARG;
    if (!slots && pool < B) return VMB_ERR_INVALID_ARG;
    if (!q || !k || !v || !g || !beta || !state || !o) return VMB_ERR_INVALID_ARG;
    const size_t es = esize(dtype);
    if (!aligned(q, es) || !aligned(k, es) || !aligned(v, es) || !aligned(g, es) || !aligned(beta, es) || !aligned(o, es) ||
        !aligned(state, 4) || !aligned(slots, 4))
        return VMB_ERR_MISALIGNED;
    if (o == q || o == k || o == v) return VMB_ERR_INVALID_ARG;
    DeltaArgs d;
    d.B = B, d.T = T, d.Hk = Hk, d.Hv = Hv, d.Dk = Dk, d.Dv = Dv;
    if ((s = delta_strides(d, strides)) != VMB_OK) return s;
    DeltaStep a{q, k, v, g, beta, state, slots, o, B, T, Hk, Hv, Dk, Dv, d.q_b, d.q_t, d.k_b, d.k_t, d.v_b, d.v_t, pool, scale, dtype};
    return launch_delta_step(a, stream);
}

vmb_status vmb_rotary_fwd(const void* q, const void* k, const float* freq, const int32_t* positions, void* q_out, void* k_out, int B,
                          int T, int Hq, int Hk, int D, int axes, const int* pairs, const int* grid, const int64_t* strides,
                          unsigned flags, vmb_dtype dtype, cudaStream_t stream) {
    if (!dtype_ok(dtype) || B < 0 || T < 0 || Hq < 0 || Hk < 0 || D < 0 || axes < 1 || axes > 4 || !pairs) return VMB_ERR_INVALID_ARG;
    if (flags & ~(VMB_ROTARY_INTERLEAVED | VMB_ROTARY_INVERSE)) return VMB_ERR_INVALID_ARG;
    long long n = 0, P = 0, cells = 1;
    if (!count(&n, {B, T, (long long)Hq + Hk, D})) return VMB_ERR_INVALID_ARG;
    RotaryArgs a{};
    for (int i = 0; i < axes; ++i) {
        if (pairs[i] < 0) return VMB_ERR_INVALID_ARG;
        P += pairs[i];
        a.pair_end[i] = (int)(P < INT_MAX ? P : INT_MAX);
        if (!positions) {
            if (!grid || grid[i] < 0 || !mul_ok(cells, grid[i], &cells)) return VMB_ERR_INVALID_ARG;
            a.grid[i] = grid[i];
        }
    }
    if (!positions && cells != T) return VMB_ERR_INVALID_ARG;
    if (P < 1 || 2 * P > D) return n == 0 && D == 0 ? VMB_OK : VMB_ERR_INVALID_ARG;
    if (n == 0) return VMB_OK;
    if (P > 4096) return VMB_ERR_UNSUPPORTED;  // (a token's sines fit the shared memory of a block)
    if (((long long)Hq + Hk) * D > INT_MAX / 4096) return VMB_ERR_UNSUPPORTED;  // (a block's vectors are counted in 32 bits)
    if (Hq > 0 && (!q || !q_out)) return VMB_ERR_INVALID_ARG;
    if (Hk > 0 && (!k || !k_out)) return VMB_ERR_INVALID_ARG;
    if (!freq) return VMB_ERR_INVALID_ARG;
    const size_t es = esize(dtype);
    if (!aligned(q, es) || !aligned(k, es) || !aligned(q_out, es) || !aligned(k_out, es) || !aligned(freq, 4) || !aligned(positions, 4))
        return VMB_ERR_MISALIGNED;
    a.q_t = (long long)Hq * D, a.k_t = (long long)Hk * D;
    a.q_b = a.q_t * T, a.k_b = a.k_t * T;
    if (strides) {
        for (int i = 0; i < 4; ++i)
            if (strides[i] < 0) return VMB_ERR_INVALID_ARG;
        // (the stride of a dimension of one has no meaning)
        const bool dense_q = (B == 1 || strides[0] == a.q_b) && (T == 1 || strides[1] == a.q_t),
                   dense_k = (B == 1 || strides[2] == a.k_b) && (T == 1 || strides[3] == a.k_t);
        if ((q && q == q_out && !dense_q) || (k && Hk && k == k_out && !dense_k)) return VMB_ERR_INVALID_ARG;
        a.q_b = strides[0], a.q_t = strides[1], a.k_b = strides[2], a.k_t = strides[3];
    }
    a.q = q, a.k = Hk > 0 ? k : nullptr, a.freq = freq, a.positions = positions, a.q_out = q_out, a.k_out = Hk > 0 ? k_out : nullptr;
    a.B = B, a.T = T, a.Hq = Hq, a.Hk = Hk, a.D = D, a.axes = axes;
    a.interleaved = (flags & VMB_ROTARY_INTERLEAVED) != 0, a.inverse = (flags & VMB_ROTARY_INVERSE) != 0, a.dtype = dtype;
    return launch_rotary(a, stream);
}

namespace {
vmb_status norm_sizes(int B, int64_t L, int C, int G, vmb_dtype dt, bool* empty) {
    long long n = 0;
    if (!dtype_ok(dt) || B < 0 || L < 0 || C < 0 || G < 0) return VMB_ERR_INVALID_ARG;
    if (!count(&n, {B, L, C})) return VMB_ERR_INVALID_ARG;
    *empty = n == 0;
    if (*empty) return VMB_OK;
    if (G < 1 || C % G) return VMB_ERR_INVALID_ARG;
    if (C > 16384 || L > (1LL << 40) || B > (1 << 24)) return VMB_ERR_UNSUPPORTED;
    return VMB_OK;
}
bool act_ok(vmb_act a) { return a == VMB_ACT_NONE || a == VMB_ACT_SILU || a == VMB_ACT_GELU; }
}  // namespace

size_t vmb_group_norm_workspace_bytes(int B, int64_t L, int C, int G, int grads, vmb_dtype dtype) {
    bool empty = false;
    if (norm_sizes(B, L, C, G, dtype, &empty) != VMB_OK) return 0;
    return empty ? 256 : norm_workspace_bytes(B, L, C, G, dtype, grads != 0);
}

vmb_status vmb_group_norm_fwd(const void* x, const float* weight, const float* bias, void* y, float* stats, int B, int64_t L, int C,
                              int G, float eps, vmb_act act, vmb_dtype dtype, void* workspace, size_t workspace_bytes,
                              cudaStream_t stream) {
    bool empty = false;
    vmb_status s = norm_sizes(B, L, C, G, dtype, &empty);
    if (s != VMB_OK) return s;
    if (!act_ok(act) || !(eps >= 0.0f)) return VMB_ERR_INVALID_ARG;
    if (empty) return VMB_OK;
    if (!x || !y || x == y) return VMB_ERR_INVALID_ARG;
    if (!aligned(x, esize(dtype)) || !aligned(y, esize(dtype)) || !aligned(weight, 4) || !aligned(bias, 4) || !aligned(stats, 8))
        return VMB_ERR_MISALIGNED;
    if ((s = check_workspace(workspace)) != VMB_OK) return s;
    NormArgs a{x, weight, bias, y, stats, B, L, C, G, eps, act, dtype};
    a.ws = workspace, a.ws_bytes = workspace_bytes;
    return launch_norm_fwd(a, stream);
}

vmb_status vmb_group_norm_bwd(const void* x, const float* weight, const float* bias, const float* stats, const void* dy, void* dx,
                              float* dweight, float* dbias, int B, int64_t L, int C, int G, vmb_act act, vmb_dtype dtype,
                              void* workspace, size_t workspace_bytes, cudaStream_t stream) {
    bool empty = false;
    vmb_status s = norm_sizes(B, L, C, G, dtype, &empty);
    if (s != VMB_OK) return s;
    if (!act_ok(act)) return VMB_ERR_INVALID_ARG;
    if (empty) return VMB_OK;
    if (!x || !stats || !dy || !dx || dx == x || dx == dy) return VMB_ERR_INVALID_ARG;
    if (!aligned(x, esize(dtype)) || !aligned(dy, esize(dtype)) || !aligned(dx, esize(dtype)) || !aligned(weight, 4) ||
        !aligned(bias, 4) || !aligned(stats, 8) || !aligned(dweight, 4) || !aligned(dbias, 4))
        return VMB_ERR_MISALIGNED;
    if ((s = check_workspace(workspace)) != VMB_OK) return s;
    NormArgs a{x, weight, bias, nullptr, const_cast<float*>(stats), B, L, C, G, 0.0f, act, dtype};
    a.dy = dy, a.dx = dx, a.dweight = dweight, a.dbias = dbias, a.ws = workspace, a.ws_bytes = workspace_bytes;
    return launch_norm_bwd(a, stream);
}

}  // extern "C"
