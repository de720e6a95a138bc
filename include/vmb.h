/*
 * vmb.h - C ABI of the GB300 (sm_103a) library for the VMamba SS2D selective
 * scan and its channel-mean variant VMeanba (arXiv 2412.16602), and for a
 * channels-last token mixer (gated delta rule, rotary positions, group norm), and for the layer
 * around a scan over tokens (projections, short causal convolution, selective scan, root-mean-square norm).
 *
 * The SS2D module (App. A, "VMamba" paragraph) is cross-scan -> selective scan
 * per direction -> cross-merge.  The selective scan is the discretised,
 * input-dependent state space model of App. A, Eqs. 3, 4 and 6.  VMeanba
 * (Sec. 2.2, Eq. 9) replaces the scan's inputs (Abar, Bbar u, C) by their mean
 * over the inner channel axis, runs one recurrence, and broadcasts the result
 * back to every channel.
 *
 * Conventions shared by every call
 *   - All tensor pointers are caller-owned DEVICE memory, dense row-major.
 *     The library allocates nothing, and scratch memory (the look-back
 *     workspace of the scans) is passed in by the caller.  The one exception
 *     is vmb_selective_scan_fwd_noalloc, for callers that cannot allocate:
 *     its scratch is a fixed array built into the library (one per device),
 *     and it keeps a host-side table of that array's device addresses.
 *   - Every call only validates its arguments and enqueues kernels on
 *     `stream`; it never synchronises (except vmb_read_status) and never
 *     throws or aborts.  Validation errors return before any launch, with no
 *     side effects.  A failed launch returns VMB_ERR_CUDA.
 *   - Shapes: B batch, K scan directions, D inner channels (d_inner), N state
 *     size (d_state), H x W the feature map, L = H*W the sequence length.
 *     A zero B, K, D, H or W is an empty problem: the call returns VMB_OK and
 *     launches nothing.  Negative sizes, or sizes whose element counts do
 *     not fit in int64, return VMB_ERR_INVALID_ARG.
 *   - dtype is the storage type of x/xs/u/delta/Bs/Cs/y/out (fp32 or bf16);
 *     A, Dskip and delta_bias are always fp32; arithmetic and the scan state
 *     are always fp32.  bf16 outputs are rounded to nearest even.
 *   - Pointers must be aligned to their element size (VMB_ERR_MISALIGNED
 *     otherwise).  16-byte aligned rows take the vectorised load path; other
 *     layouts take an element-wise path that gives the same results.
 *   - Outputs must not alias inputs.
 *   - Calls are thread-safe.  Scan calls that share one workspace must not
 *     overlap in time (order them on one stream).
 *   - Kernels are launched with programmatic stream serialization
 *     (programmatic dependent launch): their blocks may be scheduled while
 *     the previous kernel of the stream is finishing, and each waits
 *     (griddepcontrol.wait) for that kernel to complete before it reads or
 *     writes global memory.  (Two exceptions: a warp-specialised full scan or
 *     a chain of the delta rule whose grid is smaller than one wave is launched
 *     normally, so that its blocks spread over every SM; and inside the calls that start from the map,
 *     the scan's blocks that do not read the map's transpose run beside the
 *     kernel that writes it, which has itself waited for everything before the
 *     call.)  Stream order is therefore kept for any
 *     preceding work; a caller's own kernel launched after a vmb call with
 *     the same attribute must likewise wait before touching vmb outputs.
 */
#ifndef VMB_H
#define VMB_H

#include <stddef.h>
#include <stdint.h>

#include <cuda_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    VMB_OK = 0,
    VMB_ERR_INVALID_ARG = 1, /* null pointer, bad size or flag */
    VMB_ERR_MISALIGNED = 2,  /* pointer not aligned to its element size (workspace: 256 B) */
    VMB_ERR_UNSUPPORTED = 3, /* valid request this build does not implement (e.g. N > 16) */
    VMB_ERR_WORKSPACE = 4,   /* workspace missing or smaller than vmb_scan_workspace_bytes() */
    VMB_ERR_CUDA = 5,        /* a CUDA runtime call or kernel launch failed */
    VMB_ERR_TIMEOUT = 6,     /* device side: a look-back wait gave up (read via vmb_read_status) */
    VMB_ERR_BOUNDS = 7       /* device side: an index check failed (bounds-checked builds only) */
} vmb_status;

typedef enum { VMB_F32 = 0, VMB_BF16 = 1 } vmb_dtype;

/* Scan flags (bitwise OR). */
#define VMB_FLAG_SOFTPLUS 0x1u  /* delta = softplus(delta_raw + delta_bias) (Eq. 6); else raw + bias */
#define VMB_FLAG_B_ZOH 0x2u     /* Bbar = (exp(delta A) - 1) / A * B, zero-order hold (Eq. 4);
                                   else the Euler form Bbar = delta * B */
#define VMB_FLAG_SKIP_MEAN 0x4u /* vmb_mean_scan_fwd only: skip term = mean_d(Dskip_c u_d),
                                   broadcast; else per channel Dskip_c * u_d */
/* Test hook, never set in production: the first L-chunk of every sequence of
 * a multi-chunk scan does not publish its state, so that the look-back waits
 * of its successors run out (bounded, about 0.2 s) and the call reports
 * VMB_ERR_TIMEOUT through vmb_read_status; in the warp-specialised full scan
 * the first stage of every tile is never handed to the compute warps, so
 * their waits and then the copy warp's run out (bounded, about 1 s each) and
 * the call reports VMB_ERR_TIMEOUT.  No effect on other single-chunk plans. */
#define VMB_FLAG_TEST_SUPPRESS_PUBLISH 0x40000000u

/* Scan path selector for vmb_scan_workspace_bytes. */
#define VMB_PATH_FULL 0
#define VMB_PATH_MEAN 1

/*
 * vmb_cross_scan - SS2D cross-scan (App. A, "VMamba": unfold the H x W map
 * along four directions into four 1-D sequences).
 *   x   [B, D, H, W]       input map
 *   xs  [B, 4, D, L]       output sequences: direction 0 reads the map row by
 *                          row, 1 column by column, 2 and 3 are 0 and 1 reversed:
 *     xs[b,0,d,l] = x[b,d,l/W,l%W]      xs[b,1,d,l] = x[b,d,l%H,l/H]
 *     xs[b,2,d,l] = xs[b,0,d,L-1-l]     xs[b,3,d,l] = xs[b,1,d,L-1-l]
 * A pure permutation: results are bit-exact copies of x.
 */
vmb_status vmb_cross_scan(const void* x, void* xs, int B, int D, int H, int W, vmb_dtype dtype,
                          cudaStream_t stream);

/*
 * vmb_cross_merge - SS2D cross-merge (App. A, "VMamba": merge the four
 * sequence sets back into the 2-D map).
 *   ys  [B, 4, D, L]       per-direction outputs
 *   out [B, D, H, W]       out[b,d,h,w] = (ys0[p0] + ys2[p2]) + (ys1[p1] + ys3[p3]),
 *                          p0 = h*W + w, p1 = w*H + h, p2 = L-1-p0, p3 = L-1-p1,
 *                          summed in fp32 in exactly this order.
 */
vmb_status vmb_cross_merge(const void* ys, void* out, int B, int D, int H, int W,
                           vmb_dtype dtype, cudaStream_t stream);

/*
 * vmb_scan_workspace_bytes - bytes of zero-initialised device workspace that
 * vmb_selective_scan_fwd (path VMB_PATH_FULL) or vmb_mean_scan_fwd
 * (VMB_PATH_MEAN) needs for this problem on the current device, under any
 * flags and for any alignment of the tensors (the largest of the plans of the two
 * Bbar forms and of aligned and unaligned rows, which differ in tile shape and
 * chunking).  Always >= 256 (the status header).  The workspace
 * holds the status word and the chunk-carry exchange of the L-chunked scans.
 *
 * The workspace must be zero-filled once before its first use (cudaMemset or
 * a zeros tensor); afterwards every call leaves it ready for the next one.
 * Returns 0 for invalid arguments.
 */
size_t vmb_scan_workspace_bytes(int path, int B, int K, int D, int N, int H, int W,
                                vmb_dtype dtype);

/*
 * vmb_scan_kernel_count - number of kernels one vmb_selective_scan_fwd
 * (VMB_PATH_FULL) or vmb_mean_scan_fwd (VMB_PATH_MEAN) call launches for this
 * problem on the current device: 1, or 2 or 3 for the L-chunked full scans that
 * hand the chunk carry from launch to launch.  0 for an empty problem or
 * invalid arguments.  (vmb_mean_scan_merge_fwd launches the mean scan's
 * kernels plus one merge kernel.)  Bookkeeping for timing tools; the paper
 * has no counterpart.
 */
int vmb_scan_kernel_count(int path, int B, int K, int D, int N, int H, int W, vmb_dtype dtype);

/*
 * vmb_selective_scan_fwd - full-channel selective scan over K directions
 * (App. A: selection Eq. 6, discretisation Eq. 4, recurrence Eq. 3), with the
 * discretisation fused into the scan:
 *   c = k*D + d,  delta_t = softplus(delta[b,k,d,t] + delta_bias[c])
 *   h_n(-1) = 0,  h_n(t) = exp(delta_t A[c,n]) h_n(t-1) + Bbar_n(t) u[b,k,d,t]
 *   y[b,k,d,t] = sum_n Cs[b,k,n,t] h_n(t) + Dskip[c] u[b,k,d,t]
 *   u, delta, y [B, K, D, L] (dtype);  Bs, Cs [B, K, N, L] (dtype)
 *   A [K*D, N], Dskip [K*D], delta_bias [K*D] (fp32)
 *   flags: VMB_FLAG_SOFTPLUS | VMB_FLAG_B_ZOH
 *   workspace: >= vmb_scan_workspace_bytes(VMB_PATH_FULL, ...) bytes, 256-B
 *   aligned, zero-filled before first use.
 * Supports 1 <= N <= 16 (VMB_ERR_UNSUPPORTED above) and any K >= 1.
 */
vmb_status vmb_selective_scan_fwd(const void* u, const void* delta, const float* A, const void* Bs,
                                  const void* Cs, const float* Dskip, const float* delta_bias,
                                  void* y, int B, int K, int D, int N, int H, int W,
                                  unsigned flags, vmb_dtype dtype, void* workspace,
                                  size_t workspace_bytes, cudaStream_t stream);

/*
 * vmb_mean_scan_fwd - VMeanba channel-mean scan (Sec. 2.2, Eq. 9:
 * y = T^-1(Mamba(T(Abar, Bbar u, C)))), T the mean over the D channels of one
 * (batch, direction), T^-1 the broadcast back to every channel:
 *   Abar_n(t)    = (1/D) sum_d exp(delta_{d,t} A[c_d,n])      (mean after the exp)
 *   (Bbar u)_n(t)= (1/D) sum_d Bbar_{d,n}(t) u[b,k,d,t]
 *   h_n(t) = Abar_n(t) h_n(t-1) + (Bbar u)_n(t),  ybar(t) = sum_n Cs[b,k,n,t] h_n(t)
 *   y[b,k,d,t] = ybar(t) + Dskip[c] u[b,k,d,t]      (VMB_FLAG_SKIP_MEAN:
 *                ybar(t) + (1/D) sum_d Dskip[c_d] u[b,k,d,t])
 * Same arguments as vmb_selective_scan_fwd, plus
 *   ybar [B, K, L] fp32 device pointer, or NULL: optional copy of ybar.
 * The recurrence runs once per (b, k) instead of once per (b, k, d).
 * Returns VMB_ERR_UNSUPPORTED when D * L >= 2^31 (the kernel addresses one
 * (b, k) slab with 32-bit offsets).
 */
vmb_status vmb_mean_scan_fwd(const void* u, const void* delta, const float* A, const void* Bs,
                             const void* Cs, const float* Dskip, const float* delta_bias, void* y,
                             float* ybar, int B, int K, int D, int N, int H, int W, unsigned flags,
                             vmb_dtype dtype, void* workspace, size_t workspace_bytes,
                             cudaStream_t stream);

/*
 * vmb_mean_scan_grouped_fwd - grouped basis: the reduced input set I_basis of
 * Sec. 2.1 with a reduced channel dimension d = groups instead of VMeanba's
 * d = 1 (Eq. 8 counts 9BLd FLOPs for it).  The D channels of each direction
 * are split into `groups` consecutive groups of D/groups channels; T is the
 * mean over each group and T^-1 broadcasts each group's ybar to its channels:
 *   ybar[b,k,g,t] as in vmb_mean_scan_fwd over channels g*D/G .. (g+1)*D/G - 1,
 *   y[b,k,d,t] = ybar[b,k,d/(D/G),t] + Dskip[c] u[b,k,d,t] (VMB_FLAG_SKIP_MEAN:
 *   the mean of Dskip u over the group).
 * Same arguments as vmb_mean_scan_fwd plus `groups` (>= 1, divides D;
 * VMB_ERR_INVALID_ARG otherwise); ybar, if not NULL, is [B, K, groups, L]
 * fp32.  groups = 1 is vmb_mean_scan_fwd; groups = D gives the full scan's y.
 * workspace: >= vmb_scan_workspace_bytes(VMB_PATH_MEAN, B, K*groups,
 * D/groups, N, H, W, dtype) bytes (the grouped problem runs as K*groups
 * directions of D/groups channels).
 */
vmb_status vmb_mean_scan_grouped_fwd(const void* u, const void* delta, const float* A, const void* Bs,
                                     const void* Cs, const float* Dskip, const float* delta_bias,
                                     void* y, float* ybar, int B, int K, int D, int N, int H, int W,
                                     int groups, unsigned flags, vmb_dtype dtype, void* workspace,
                                     size_t workspace_bytes, cudaStream_t stream);

/*
 * vmb_mean_scan_merge_fwd - the channel-mean path of an SS2D block (Sec. 2.2,
 * Eq. 9, then the App. A cross-merge) with the broadcast T^-1 fused into the
 * merge, so the per-channel output y [B, 4, D, L] is never written:
 *   every direction's u at the position it merges into is the map itself,
 *   u_k[b,d,p_k(h,w)] = x[b,d,h,w], hence
 *   out[b,d,h,w] = (y0 + y2) + (y1 + y3),
 *   y_k = ybar_k[b, p_k] + Dskip[k*D+d] x[b,d,h,w]  (p_k as in vmb_cross_merge;
 *         VMB_FLAG_SKIP_MEAN: y_k = ybar_k[b, p_k] + the mean skip term of k)
 *   u (= vmb_cross_scan(x)), delta [B, 4, D, L], Bs, Cs [B, 4, N, L] (dtype);
 *   A [4*D, N], Dskip [4*D], delta_bias [4*D] (fp32);
 *   x, out [B, D, H, W] (dtype), out must not alias x;
 *   ybar [B, 4, L] fp32, required: receives ybar_k(t) (plus the broadcast mean
 *   skip term under VMB_FLAG_SKIP_MEAN) and is read back by the merge.
 *   workspace: as vmb_mean_scan_fwd with K = 4 (VMB_PATH_MEAN).
 * The same fp32 operations in the same order as vmb_cross_merge applied to
 * vmb_mean_scan_fwd's y, so fp32 results are bit-identical to that unfused
 * pair; bf16 storage rounds once, at the end (the unfused pair rounds y
 * first).  Not in the paper as such: its kernels keep the steps apart.
 */
vmb_status vmb_mean_scan_merge_fwd(const void* u, const void* delta, const float* A, const void* Bs,
                                   const void* Cs, const float* Dskip, const float* delta_bias,
                                   const void* x, void* out, float* ybar, int B, int D, int N, int H,
                                   int W, unsigned flags, vmb_dtype dtype, void* workspace,
                                   size_t workspace_bytes, cudaStream_t stream);

/*
 * vmb_ss2d_full_fwd - the scan side of a full-channel SS2D block in one call
 * (App. A: cross-scan, the selective scan of Eqs. 3, 4 and 6, cross-merge)
 * without the cross-scanned sequences xs [B, 4, D, L] being written:
 *   y   = vmb_selective_scan_fwd(vmb_cross_scan(x), delta, ...) with K = 4,
 *   out = vmb_cross_merge(y)
 *   x, out [B, D, H, W] (dtype); y [B, 4, D, L] (dtype), written (the
 *   per-direction output); xt [B, D, W, H] (dtype), caller-owned scratch
 *   (overwritten); none of x, xt, y, out may alias another;
 *   delta [B, 4, D, L], Bs, Cs [B, 4, N, L] (dtype); A [4*D, N], Dskip [4*D],
 *   delta_bias [4*D] (fp32); flags and workspace as vmb_selective_scan_fwd with
 *   K = 4 (vmb_scan_workspace_bytes(VMB_PATH_FULL, B, 4, D, N, H, W, dtype)).
 * Short maps of 9 to 16 states (up to 256 pixels, by the number of channel rows) take one
 * launch that reads the map in every direction's order and merges on chip; xt
 * is then left as it was.  Where the warp-specialised scan kernel runs (rows of
 * 16-byte multiples, 16-byte aligned tensors, enough channel rows) direction k's step
 * l reads the value the cross-scan would have put there: directions 0 and 2
 * the (b, d) planes of x row by row (forward and reversed), directions 1 and 3
 * the rows of xt, the transpose of every plane (written by this call), so the
 * map moves 2 B*D*L elements instead of the cross-scan's 5 B*D*L.  Otherwise
 * the cross-scan is written into y and the scan runs in place.  Either way
 * the values and operations are those of the three separate calls, so y and
 * out are bit-identical to them.  Not in the paper as such: its kernels keep
 * the steps apart.
 */
vmb_status vmb_ss2d_full_fwd(const void* x, void* xt, const void* delta, const float* A,
                             const void* Bs, const void* Cs, const float* Dskip,
                             const float* delta_bias, void* y, void* out, int B, int D, int N,
                             int H, int W, unsigned flags, vmb_dtype dtype, void* workspace,
                             size_t workspace_bytes, cudaStream_t stream);

/*
 * vmb_ss2d_mean_fwd - the scan side of a VMeanba SS2D block in one call: the
 * App. A cross-scan, the channel-mean scan (Sec. 2.2, Eq. 9) and the App. A
 * cross-merge, without the cross-scanned sequences xs [B, 4, D, L] or the
 * per-channel output y ever being written.  Direction k's step l reads the
 * value the cross-scan would have put there: directions 0 and 2 read the
 * (b, d) planes of x row by row (forward and reversed), directions 1 and 3 the
 * rows of xt, the transpose of every plane (xt[b,d,w,h] = x[b,d,h,w], written
 * by this call); the merge applies the broadcast and the skip term:
 *   out = vmb_mean_scan_merge_fwd(vmb_cross_scan(x), delta, ..., x)
 *   x, out [B, D, H, W] (dtype), out must not alias x;
 *   xt [B, D, W, H] (dtype), caller-owned scratch (overwritten), aliasing
 *   neither x nor out;
 *   delta [B, 4, D, L], Bs, Cs [B, 4, N, L] (dtype); A [4*D, N], Dskip [4*D],
 *   delta_bias [4*D] (fp32); ybar [B, 4, L] fp32, required (as in
 *   vmb_mean_scan_merge_fwd); flags and workspace as vmb_mean_scan_fwd with
 *   K = 4 (vmb_scan_workspace_bytes(VMB_PATH_MEAN, B, 4, D, N, H, W, dtype)).
 * Moves 2 B*D*L elements for the map instead of the cross-scan's 5 B*D*L.
 * The same fp32 operations in the same order as that pair of calls, so fp32
 * results are bit-identical to it.  Not in the paper as such: its kernels keep
 * the steps apart.
 */
vmb_status vmb_ss2d_mean_fwd(const void* x, void* xt, const void* delta, const float* A,
                             const void* Bs, const void* Cs, const float* Dskip,
                             const float* delta_bias, void* out, float* ybar, int B, int D, int N,
                             int H, int W, unsigned flags, vmb_dtype dtype, void* workspace,
                             size_t workspace_bytes, cudaStream_t stream);

/*
 * vmb_selective_scan_fwd_noalloc - vmb_selective_scan_fwd for callers that
 * cannot allocate device memory (for example plugin code inside a framework
 * whose memory pool owns the device and forbids allocations of its own, or a
 * serving loop that must not allocate once it runs).  The paper has no
 * counterpart; this is a deployment convenience.
 *   Same arguments and results as vmb_selective_scan_fwd, without the
 *   workspace: the chunk-exchange scratch is a 16 MiB array built into the
 *   library, which every GPU that loads libvmb holds until the process exits.
 *   The call allocates nothing.
 *   Every argument check runs first: a rejected call queues nothing.
 *   Returns VMB_ERR_WORKSPACE when this call's plan (problem and flags) needs
 *   more than 16 MiB of scratch; vmb_scan_workspace_bytes(VMB_PATH_FULL, ...)
 *   <= 16 MiB guarantees that it does not.
 *   The first call made with a given device current looks up the array's
 *   device address on that device and keeps it for the life of the process;
 *   make that first call before any stream capture, and do not use this
 *   entry point across a cudaDeviceReset of that device.  Each call first
 *   clears the part of the array that must start at zero (an asynchronous
 *   memset on `stream`).  All calls share the one array per device, so calls
 *   that overlap in time on the GPU (other streams, other host threads) race
 *   and must be serialised by the caller.  Device-side wait timeouts have no
 *   readback for this entry point.
 */
vmb_status vmb_selective_scan_fwd_noalloc(const void* u, const void* delta, const float* A,
                                          const void* Bs, const void* Cs, const float* Dskip,
                                          const float* delta_bias, void* y, int B, int K, int D,
                                          int N, int H, int W, unsigned flags, vmb_dtype dtype,
                                          cudaStream_t stream);

/*
 * The paper's own kernel setting (Sec. 4, "Kernel Implementation"): the
 * discretisation runs outside the scan kernel, which reads the materialised
 * operands Abar and Bbar u.  These three calls reproduce that split, for
 * measuring it next to the fused scans above; they are not needed to compute
 * the SS2D output.  Operands are fp32; their sizes grow with N (a B=1 VMamba-T
 * stage-1 map with N = 16 materialises 2 x 154 MB).
 *
 * vmb_discretise_fwd - Eqs. 4 and 6 for every (b, k, d, n, l):
 *   delta = softplus(delta_raw + delta_bias[c]) (or raw + bias without
 *   VMB_FLAG_SOFTPLUS), dA[b,k,d,n,l] = exp(delta A[c,n]),
 *   dBu[b,k,d,n,l] = delta B[b,k,n,l] u[b,k,d,l] (Euler) or
 *   (exp(delta A) - 1) / A B u under VMB_FLAG_B_ZOH.
 *   u, delta [B,K,D,L], Bs [B,K,N,L] in dtype; A [K*D,N], delta_bias [K*D] fp32;
 *   dA, dBu [B,K,D,N,L] fp32 out.  flags: VMB_FLAG_SOFTPLUS | VMB_FLAG_B_ZOH.
 *   N in 1..16 (VMB_ERR_UNSUPPORTED above).
 *
 * vmb_discretise_mean_fwd - Eq. 9's T applied to the discretised operands:
 *   dAm[b,k,n,l] = mean_d exp(delta_d A[c_d,n]),
 *   dBum[b,k,n,l] = mean_d Bbar[b,k,d,n,l] u[b,k,d,l], fp32 [B,K,N,L] out (the
 *   [B,K,1,N,L] operands of the scan kernel).  Same inputs and flags as above.
 *
 * vmb_scan_only_fwd - Eq. 3 without the skip term on materialised operands of
 *   Dm channels per (b, k) (Dm = D for the full path, 1 after the mean):
 *   h[n] = dA h[n] + dBu from h = 0, y[b,k,d,l] = sum_n Cs[b,k,n,l] h[n].
 *   dA, dBu [B,K,Dm,N,L] fp32, Cs [B,K,N,L] in dtype, y [B,K,Dm,L] fp32 out.
 *   Deterministic; no workspace.  N in 1..16.
 */
vmb_status vmb_discretise_fwd(const void* u, const void* delta, const float* A, const void* Bs,
                              const float* delta_bias, float* dA, float* dBu, int B, int K, int D,
                              int N, int H, int W, unsigned flags, vmb_dtype dtype,
                              cudaStream_t stream);
vmb_status vmb_discretise_mean_fwd(const void* u, const void* delta, const float* A, const void* Bs,
                                   const float* delta_bias, float* dAm, float* dBum, int B, int K,
                                   int D, int N, int H, int W, unsigned flags, vmb_dtype dtype,
                                   cudaStream_t stream);
vmb_status vmb_scan_only_fwd(const float* dA, const float* dBu, const void* Cs, float* y, int B,
                             int K, int Dm, int N, int H, int W, vmb_dtype dtype,
                             cudaStream_t stream);

/*
 * vmb_selection_fwd - the selection functions of Eq. 6 (App. A): B, C and the
 * raw Delta of every step as linear maps of the scan input over the D channels
 * of that step and direction, with per-direction weights:
 *   Bs[b,k,n,l] = sum_d WB[k,n,d] u[b,k,d,l]      s_B = Linear_N(u)
 *   Cs[b,k,n,l] = sum_d WC[k,n,d] u[b,k,d,l]      s_C = Linear_N(u)
 *   z_r = sum_d Wz[k,r,d] u[b,k,d,l],  delta_raw[b,k,d,l] = sum_r Wup[k,d,r] z_r
 * The Delta branch is a rank-R map; R = 1 with Wup = 1 is the printed
 * s_Delta = Broadcast_D(Linear_1(u)).  The scans then apply
 * Delta = softplus(delta_raw + delta_bias) (VMB_FLAG_SOFTPLUS).
 *   u [B,K,D,L] (dtype); WB, WC [K,N,D], Wz [K,R,D], Wup [K,D,R] fp32;
 *   Bs, Cs [B,K,N,L], delta_raw [B,K,D,L] (dtype) out.  N and R in 1..16
 *   (VMB_ERR_UNSUPPORTED above).  Accumulation in fp32 (channels in order).
 */
vmb_status vmb_selection_fwd(const void* u, const float* WB, const float* WC, const float* Wz,
                             const float* Wup, void* Bs, void* Cs, void* delta_raw, int B, int K,
                             int D, int N, int R, int H, int W, vmb_dtype dtype, cudaStream_t stream);

/*
 * The selection functions with the Delta branch left in its low-rank form
 * (Eq. 6, App. A: s_Delta = Linear_D(Linear_R(u))), so the raw Deltas
 * [B,K,D,L] are never written: the scan expands them itself.
 *
 * vmb_selection_lowrank_fwd - as vmb_selection_fwd, but writes the rank-R
 *   intermediate z[b,k,r,l] = sum_d Wz[k,r,d] u[b,k,d,l] (fp32 [B,K,R,L],
 *   4-byte aligned) instead of delta_raw; no Wup.  Bs, Cs as there.
 *
 * vmb_selective_scan_lowrank_fwd - vmb_selective_scan_fwd with
 *   delta_raw[b,k,d,l] = sum_r Wup[k,d,r] z[b,k,r,l] (r in order, fp32)
 *   formed inside the scan from z [B,K,R,L] fp32 and Wup [K,D,R] fp32 (R in
 *   1..16; VMB_ERR_UNSUPPORTED above); every other argument, flag and the
 *   workspace (vmb_scan_workspace_bytes(VMB_PATH_FULL, ...)) as there; y must
 *   not alias u.  The warp-specialised scan (9 to 16 states, rows of 16-byte
 *   multiples, 16-byte aligned tensors, enough channel rows, Euler Bbar) reads
 *   z instead of the raw Deltas, i.e. R instead of D values per step and
 *   direction; for other plans the raw Deltas are written into y (rounded to
 *   the storage type) and the scan runs in place.  In fp32 the result is
 *   bit-identical to vmb_selection_fwd's raw Deltas fed to
 *   vmb_selective_scan_fwd; with bf16 storage the warp-specialised scan keeps
 *   the raw Deltas in fp32 (that pair rounds them to bf16 first).
 */
vmb_status vmb_selection_lowrank_fwd(const void* u, const float* WB, const float* WC, const float* Wz,
                                     void* Bs, void* Cs, float* z, int B, int K, int D, int N, int R, int H,
                                     int W, vmb_dtype dtype, cudaStream_t stream);
vmb_status vmb_selective_scan_lowrank_fwd(const void* u, const float* z, const float* Wup, const float* A,
                                          const void* Bs, const void* Cs, const float* Dskip,
                                          const float* delta_bias, void* y, int B, int K, int D, int N,
                                          int R, int H, int W, unsigned flags, vmb_dtype dtype,
                                          void* workspace, size_t workspace_bytes, cudaStream_t stream);

/*
 * vmb_mean_scan_lowrank_fwd - vmb_mean_scan_fwd (the channel-mean scan of
 *   Sec. 2.2, Eq. 9) with delta_raw = Wup z formed inside the scan, as in
 *   vmb_selective_scan_lowrank_fwd: z [B,K,R,L] fp32, Wup [K,D,R] fp32, R in
 *   1..16; every other argument (ybar optional), flag and the workspace
 *   (vmb_scan_workspace_bytes(VMB_PATH_MEAN, ...)) as vmb_mean_scan_fwd; y
 *   must not alias u.  For ranks up to 8 with the Euler Bbar each thread of
 *   the reduction forms the raw Delta of its step and channel (R FMAs) instead
 *   of reading it; otherwise the raw Deltas are written into y (rounded to the
 *   storage type) and the scan runs in place.  In fp32 the result is
 *   bit-identical to vmb_selection_fwd's raw Deltas fed to vmb_mean_scan_fwd.
 */
vmb_status vmb_mean_scan_lowrank_fwd(const void* u, const float* z, const float* Wup, const float* A,
                                     const void* Bs, const void* Cs, const float* Dskip,
                                     const float* delta_bias, void* y, float* ybar, int B, int K, int D,
                                     int N, int R, int H, int W, unsigned flags, vmb_dtype dtype,
                                     void* workspace, size_t workspace_bytes, cudaStream_t stream);

/*
 * vmb_mean_scan_train_fwd - vmb_mean_scan_grouped_fwd (groups = 1: the
 * channel-mean scan of Eq. 9) that also keeps, for vmb_mean_scan_bwd, the
 * group means it forms on the way:
 *   saved [B, K, groups, N + 1, L] fp32 out: rows n < N are Abar_n(t) (the
 *   mean of exp(delta A) over the group), row N is the mean of delta u.
 * The backward then skips recomputing them (N exponentials per element).
 * Same arguments and workspace as vmb_mean_scan_grouped_fwd plus `saved`
 * (not NULL, 4-byte aligned, 16-byte aligned for the backward's vector
 * loads); flags: VMB_FLAG_SOFTPLUS only (the backward covers Euler Bbar and
 * the per-channel skip term: VMB_FLAG_B_ZOH and VMB_FLAG_SKIP_MEAN give
 * VMB_ERR_UNSUPPORTED).  y and ybar are the grouped forward's, bit for bit.
 */
vmb_status vmb_mean_scan_train_fwd(const void* u, const void* delta, const float* A, const void* Bs,
                                   const void* Cs, const float* Dskip, const float* delta_bias,
                                   void* y, float* ybar, float* saved, int B, int K, int D, int N,
                                   int H, int W, int groups, unsigned flags, vmb_dtype dtype,
                                   void* workspace, size_t workspace_bytes, cudaStream_t stream);

/*
 * vmb_mean_scan_bwd - gradients of the channel-mean scan (Sec. 2.2, Eq. 9) or,
 * with groups > 1, of the grouped basis (Sec. 2.1, Eq. 8; vmb_mean_scan_grouped_fwd),
 * for the Euler Bbar and the per-channel skip term: the reverse-mode
 * derivative of the forward, given gy = dLoss/dy [B, K, D, L] (dtype).  Per
 * sequence (b, k, group) the states are recomputed forward, the adjoint
 *   lam_n(t) = C_n(t) sum_d gy_d(t) + Abar_n(t+1) lam_n(t+1)
 * runs backward in time, and the chain rule goes through the group mean and
 * the softplus.  Outputs (every one written, none accumulated into):
 *   gu, gdelta [B, K, D, L] (dtype): d/du and d/d(raw delta);
 *   gA [K*D, N], gDskip [K*D], gdelta_bias [K*D] (fp32), summed over the batch;
 *   gBs, gCs [B, K, N, L] (dtype), summed over the groups of each (b, k).
 * Same inputs as vmb_mean_scan_grouped_fwd (delta is the raw Delta); flags:
 * VMB_FLAG_SOFTPLUS (VMB_FLAG_B_ZOH and VMB_FLAG_SKIP_MEAN: VMB_ERR_UNSUPPORTED).
 * saved: the means vmb_mean_scan_train_fwd wrote for the same inputs,
 * groups and flags (4-byte aligned), or NULL to recompute them here.
 * workspace: >= vmb_mean_scan_bwd_workspace_bytes(...) bytes, 256-B aligned,
 * any contents (the group means, chunk carries and adjoints of every
 * sequence, fp32: about 2 x (N + 2) x 4 bytes per (b, k, group, step)).  Every
 * reduction runs in a fixed order: results are deterministic.  The paper
 * trains no VMeanba layer (it replaces layers of a trained model); this is the
 * chain rule of the forward defined there.
 */
vmb_status vmb_mean_scan_bwd(const void* u, const void* delta, const float* A, const void* Bs,
                             const void* Cs, const float* Dskip, const float* delta_bias,
                             const void* gy, const float* saved, void* gu, void* gdelta, float* gA,
                             void* gBs, void* gCs, float* gDskip, float* gdelta_bias, int B, int K,
                             int D, int N, int H, int W, int groups, unsigned flags,
                             vmb_dtype dtype, void* workspace, size_t workspace_bytes,
                             cudaStream_t stream);
size_t vmb_mean_scan_bwd_workspace_bytes(int B, int K, int D, int N, int H, int W, int groups,
                                         vmb_dtype dtype);

/*
 * A channels-last token mixer over maps and videos: the gated delta rule (the recurrence over
 * tokens with a matrix state, next to the diagonal one of the scans above), rotary positions with
 * several axes for its queries and keys, and group norm with an activation.  None of the three is
 * in the paper.  Activations have the storage type `dtype`; states, norm weights, their gradients
 * and statistics are fp32, and so is all arithmetic.  Tokens (pixels) come before heads
 * (channels).  A workspace of these calls serves them alone (not the scans, and the
 * delta rule's not the norm); vmb_read_status reads its status word.
 *
 * vmb_delta_rule_fwd - the gated delta rule, from S_0 = initial_state (zeros if NULL), per
 * sequence and value head, S [Dk, Dv], a_t = exp(g_t):
 *     S_t = a_t (I - beta_t k_t k_t^T) S_{t-1} + beta_t k_t v_t^T,   o_t = scale S_t^T q_t
 * (the state is decayed, what it returns for k_t is corrected towards v_t, then it is read),
 * computed in chunks of 64 tokens.
 *   q, k [B, T, Hk, Dk], v [B, T, Hv, Dv], g, beta [B, T, Hv], o [B, T, Hv, Dv] (dtype); Hv is a
 *   multiple of Hk, value head h reads key head h / (Hv / Hk); initial_state, final_state
 *   [B, Hv, Dk, Dv] fp32, either may be NULL; they may not overlap.
 *   strides: NULL (dense), or six host values: the elements between batch rows and between tokens
 *   of q, of k and of v (parts of one projection's output); heads and channels are dense.
 *   offsets: NULL, or int32 [B + 1] on the device: B packed sequences, sequence b is rows
 *   offsets[b] .. offsets[b + 1] - 1 of `total` tokens (the batch dimension of the tensors is
 *   then 1, T a bound of the longest sequence, as loose as INT_MAX, batch strides unused).  Without offsets total is
 *   B * T.  Offsets that decrease, leave [0, total] or give a sequence longer than T are cut to
 *   what is in range and reported as VMB_ERR_BOUNDS by vmb_read_status; rows that no sequence
 *   holds (the padding of a token buffer) are zero in o and in the gradients.
 *   saved: NULL, or vmb_delta_rule_saved_bytes(...) bytes (16-byte aligned) that receive the
 *   state before each chunk and the residuals v_t - S^T k_t, for vmb_delta_rule_bwd.
 *   Keys of length above one with beta near one let the state grow, as the recurrence does.
 *   g = -inf forgets the state exactly.  What is not finite in a token reaches the tokens after it,
 *   as the recurrence has it, and no more than the 15 before it (those of its block of 16).  Dk in
 *   1..128 (VMB_ERR_UNSUPPORTED above), any Dv >= 1.
 *   workspace: >= vmb_delta_rule_workspace_bytes(..., grads = 0, ...) bytes, 256-byte aligned, the
 *   first 256 zero-filled before its first use.
 *   Rounding: with bf16 storage q, k, v and dout enter the products as they are, and what is computed
 *   (states, residuals, the decayed products of keys and queries) as the sum of two bf16 values (16
 *   bits), except that S^T q, which only o sees, takes the state's leading term; with fp32 storage
 *   every operand is the sum of two tf32 values (22 bits; a product is off by 7.2e-7 at most).  Sums,
 *   states and decays are fp32.  What is kept in `saved`, and what the reverse pass hands on per
 *   chunk, has the storage type.
 *
 * vmb_delta_rule_bwd - the gradients, given dout = dLoss/do [B, T, Hv, Dv] and dfinal_state =
 * dLoss/dS_T (or NULL): dq, dk, dv, dg, dbeta (shapes and type of the inputs, dense) and
 * dinitial_state (fp32; NULL: not wanted).  saved: what the forward kept for the same inputs.  The
 * gradients of a key head are summed over its value heads in order.  Deterministic.
 *
 * vmb_delta_rule_step - T tokens (a few) per sequence from the states in `state` [pool, Hv, Dk, Dv]
 * fp32, updated in place: serving.  slots: NULL (row b uses state b; pool >= B), or int32 [B] on
 * the device: the state of row b; rows whose slot is outside [0, pool) have none: their o is
 * zero.  Slots in use are distinct.  The other arguments as above.  No workspace.
 */
size_t vmb_delta_rule_workspace_bytes(int B, int T, int64_t total, int packed, int Hk, int Hv, int Dk, int Dv,
                                      int grads, vmb_dtype dtype);
size_t vmb_delta_rule_saved_bytes(int B, int T, int64_t total, int packed, int Hv, int Dk, int Dv, vmb_dtype dtype);
vmb_status vmb_delta_rule_fwd(const void* q, const void* k, const void* v, const void* g, const void* beta,
                              const int64_t* strides, const float* initial_state, const int32_t* offsets,
                              void* o, float* final_state, void* saved, int B, int T, int64_t total, int Hk,
                              int Hv, int Dk, int Dv, float scale, vmb_dtype dtype, void* workspace,
                              size_t workspace_bytes, cudaStream_t stream);
vmb_status vmb_delta_rule_bwd(const void* q, const void* k, const void* g, const void* beta,
                              const int64_t* strides, const int32_t* offsets, const void* dout,
                              const float* dfinal_state, const void* saved, void* dq, void* dk, void* dv,
                              void* dg, void* dbeta, float* dinitial_state, int B, int T, int64_t total,
                              int Hk, int Hv, int Dk, int Dv, float scale, vmb_dtype dtype, void* workspace,
                              size_t workspace_bytes, cudaStream_t stream);
vmb_status vmb_delta_rule_step(const void* q, const void* k, const void* v, const void* g, const void* beta,
                               const int64_t* strides, float* state, const int32_t* slots, void* o, int B,
                               int T, int Hk, int Hv, int Dk, int Dv, int pool, float scale, vmb_dtype dtype,
                               cudaStream_t stream);

/*
 * vmb_rotary_fwd - rotary positions with several axes (time, row, column, ...): the first 2P
 * channels of every head are P pairs, pair i is turned by the angle p f_i, p the token's position
 * on the pair's axis:  (x, y) -> (x cos - y sin, y cos + x sin); the other channels are copied.
 *   q [B, T, Hq, D], k [B, T, Hk, D] or NULL (Hk = 0), q_out, k_out dense (dtype); an output may
 *   be its (dense) input, otherwise outputs do not overlap inputs.
 *   freq [P] fp32 (angle per position, of every pair); axes in 1..4; pairs[axes] (host): the
 *   pairs of each axis, in the order of the channels, P their sum, 1 <= P, 2P <= D;
 *   positions int32 [axes, B, T] on the device, or NULL: grid[axes] (host), whose product is T:
 *   token t lies at its row-major place in that grid (a map: {H, W}; a video: {frames, H, W}).
 *   strides: NULL (dense), or four host values: the elements between batch rows and between tokens
 *   of q and of k.
 *   flags: VMB_ROTARY_INTERLEAVED: pair i is channels (2i, 2i + 1), otherwise (i, i + P);
 *          VMB_ROTARY_INVERSE: the opposite angle, which is the gradient with respect to q and k.
 * Angles carry an error of about 2^-24 of a turn at any position (not 2^-24 of the angle).
 */
#define VMB_ROTARY_INTERLEAVED 0x1u
#define VMB_ROTARY_INVERSE 0x2u
vmb_status vmb_rotary_fwd(const void* q, const void* k, const float* freq, const int32_t* positions,
                          void* q_out, void* k_out, int B, int T, int Hq, int Hk, int D, int axes,
                          const int* pairs, const int* grid, const int64_t* strides, unsigned flags,
                          vmb_dtype dtype, cudaStream_t stream);

/*
 * vmb_group_norm_fwd - group norm with an activation, channels last:
 *   y = act(weight n + bias), n = (x - mean) rstd, mean and variance over the L pixels and the
 *   C / G channels of a group, rstd = 1 / sqrt(variance + eps).
 *   x, y [B, L, C] (dtype); weight, bias [C] fp32 or NULL (1 and 0); stats [B, G, 2] fp32 (mean,
 *   rstd) or NULL.  G divides C; C <= 16384 (VMB_ERR_UNSUPPORTED above).
 * vmb_group_norm_bwd - its gradients given dy [B, L, C]: dx (dtype), dweight, dbias [C] fp32
 *   (either may be NULL); stats: the forward's.  Sums in a fixed order: deterministic (rows that are
 *   not 16-byte aligned are summed in another order than aligned ones).
 *   workspace: >= vmb_group_norm_workspace_bytes(...) bytes, 256-byte aligned, all of it
 *   zero-filled before its first use; calls that share one must not overlap in time.
 */
typedef enum { VMB_ACT_NONE = 0, VMB_ACT_SILU = 1, VMB_ACT_GELU = 2 } vmb_act; /* GELU: z Phi(z), Phi the normal distribution */
size_t vmb_group_norm_workspace_bytes(int B, int64_t L, int C, int G, int grads, vmb_dtype dtype);
vmb_status vmb_group_norm_fwd(const void* x, const float* weight, const float* bias, void* y, float* stats,
                              int B, int64_t L, int C, int G, float eps, vmb_act act, vmb_dtype dtype,
                              void* workspace, size_t workspace_bytes, cudaStream_t stream);
vmb_status vmb_group_norm_bwd(const void* x, const float* weight, const float* bias, const float* stats,
                              const void* dy, void* dx, float* dweight, float* dbias, int B, int64_t L,
                              int C, int G, vmb_act act, vmb_dtype dtype, void* workspace,
                              size_t workspace_bytes, cudaStream_t stream);

/*
 * ---------------------------------------------------------------- a layer around a scan over tokens
 *
 * The operators of a state space layer over sequences of tokens (App. A's selective scan, Eqs. 3
 * and 6, without the map's directions): the projections, the short causal convolution, the scan
 * with its gate, and the norm before them.  Channels last: x [B, T, C].  Activations have the storage
 * type `dtype`; filters, A, D, biases, norm weights, the states of the scan and the gradients of all these are fp32,
 * and so is all arithmetic, with the device's approximate exponential (2^-22) and reciprocal in SiLU, softplus
 * and the decays.
 *   strides: NULL (dense), or host values, two for each tensor: the elements between batch rows and
 *   between tokens (parts of one projection's output); channels are dense.
 *   offsets: NULL, or int32 [B + 1] on the device: B packed sequences, sequence b is rows
 *   offsets[b] .. offsets[b + 1] - 1 of `total` tokens (the batch dimension is then 1; T and batch
 *   strides are unused).  Without offsets total is B * T.  Offsets that leave [0, total] are cut to what is in
 *   range; where they decrease, what a call writes for the sequences and rows concerned is undefined, but in range.  The
 *   scan and, where there are tokens, its gradients report both as VMB_ERR_BOUNDS through vmb_read_status.  Rows that no sequence holds are
 *   zero in the outputs and in the gradients.
 *   slots: NULL (row b uses state b; pool >= B), or int32 [B] on the device: the state of row b; rows
 *   whose slot is outside [0, pool) have none: their outputs are zero.  Slots in use are distinct.
 *   At most 2^30 - 1 tokens, 2^24 sequences and 2^22 channels (VMB_ERR_UNSUPPORTED above), and for the
 *   scan and the gradients of the convolution fewer than 2^24 elements between tokens.
 *   Gradients are deterministic: sums in a fixed order.  Those of an empty problem (no tokens, rows or channels) are
 *   written too, as zeros, where they have elements: sums of nothing.
 *   Workspaces are 256-byte aligned, the first 256 bytes zero-filled before the first use; calls that
 *   share one must not overlap in time.
 *
 * vmb_causal_conv_fwd - a filter of W taps for each channel along the tokens of a sequence:
 *     z_t = bias + sum_j weight_j x_(t - W + 1 + j),   y_t = act(z_t)
 *   with initial_state [B, W - 1, C] (dtype; NULL: zeros) before a sequence's first token.
 *   weight [C, W] fp32, bias [C] fp32 or NULL, y [B, T, C] dense, final_state [B, W - 1, C] (dtype) or
 *   NULL: the last W - 1 inputs of each sequence, of the initial state where it is shorter.
 *   W in 1..4 (VMB_ERR_UNSUPPORTED above); act: VMB_ACT_NONE or VMB_ACT_SILU.
 * vmb_causal_conv_bwd - given dy (dense) and dfinal_state (or NULL): dx [B, T, C] dense (dtype), dweight,
 *   dbias (fp32; NULL: not wanted), dinitial_state (dtype; NULL: not wanted).
 * vmb_causal_conv_step - T tokens (a few) of every row, `state` [pool, W - 1, C] (dtype) updated in place.
 *
 * vmb_token_scan_fwd - the selective scan of every channel, from h_0 = initial_state [B, D, N] fp32
 * (NULL: zeros):
 *     dt = softplus(delta + delta_bias)  (VMB_FLAG_SOFTPLUS; otherwise delta + delta_bias),
 *     h_t = exp(dt A) h_(t-1) + dt B_t x_t,   y_t = (C_t . h_t + D x_t) silu(z_t)
 *   x, delta, z [B, T, D], Bm, Cm [B, T, N] (dtype; z NULL: no gate), A [D, N], Dskip, delta_bias [D] fp32
 *   (the latter two may be NULL); strides: ten values, of x, delta, Bm, Cm, z; y [B, T, D] dense,
 *   final_state [B, D, N] fp32 or NULL.  N in 1..16 (VMB_ERR_UNSUPPORTED above).
 *   saved: NULL, or vmb_token_scan_saved_bytes(...) bytes (16-byte aligned) for the state before every
 *   16 tokens, which vmb_token_scan_bwd takes.
 *   A decay is taken as 2^(dt A'), A' = A log2 e rounded to fp32: off by 2^-22 and 2^-23 |dt A| of itself, and
 *   over a segment of a cut sequence (64 tokens or more) as the power of the sum of its step sizes.  Outputs, states
 *   and gradients are off by that over the tokens that a state remembers, more than a recurrence in fp32 with a full
 *   exponential.  Where dt A is positive and its sum over a segment passes 88, they may be infinite or NaN though
 *   the recurrence token by token is finite.
 * vmb_token_scan_bwd - given dy (dense) and dfinal_state (or NULL): dx, ddelta, dBm, dCm, dz (shapes of the
 *   inputs, dense, dtype; dz where z is), dA, dDskip, ddelta_bias, dinitial_state (fp32; the last three may be NULL).
 * vmb_token_scan_step - T tokens (a few) of every row, `state` [pool, D, N] fp32 updated in place.
 *
 * vmb_rms_norm_fwd - rows of C channels:  s = x + residual (rounded to dtype; s = x without one),
 *     y = s rstd weight,  rstd = 1 / sqrt(mean(s^2) + eps)
 *   x, residual (or NULL), sum (with a residual) [rows, C] dense (dtype), weight [C] fp32 or NULL (1).
 *   scale NULL: y [rows, C] (dtype).  scale [rows] fp32: y holds 8-bit e4m3 values whose products with
 *   their row's scale are the norm's output: scale = max |y| / 448, 2^-100 at least.
 *   rstd [rows] fp32 or NULL.  Squares are summed in fp32: values are below 2^57.  C <= 8192 (VMB_ERR_UNSUPPORTED
 *   above); rows of no channels have no scale and no rstd (VMB_ERR_INVALID_ARG where one is wanted).
 * vmb_rms_norm_bwd - given dy, and dsum (or NULL), the gradient that reaches s on its own: dx [rows, C], the
 *   gradient of x and of the residual alike, and dweight [C] fp32 (or NULL).  x: what was normalised (the forward's sum,
 *   if it had a residual); rstd: the forward's.
 *
 * vmb_linear_fwd - matrix product with the epilogue of a projection:
 *     z = x weight^T + bias,   y = act(z) + residual
 *   x [M, K] (x_stride elements between its rows), weight [N, K] dense, bias [N] fp32 or NULL, residual
 *   [M, N] bf16 or NULL, y [M, N] bf16, pre [M, N] bf16 or NULL: z, for vmb_linear_bwd.
 *   x_scale, weight_scale: both NULL: x and weight are bf16; x_scale [M] and weight_scale [N] fp32: they are e4m3
 *   values to be multiplied by the scale of their row (what vmb_rms_norm_fwd writes in 8 bits).
 *   Products are exact and summed in fp32 by the tensor cores; one rounding, to y.  SiLU and GELU keep 12 bits, also
 *   where they are small (below 2^-119 they may be zero).  Any K, N and x_stride; rows of whole vectors of 16 bytes (K, x_stride and, for the gradients, N multiples of 8;
 *   16 with e4m3) take the fast kernels.  Waits of the kernels are bounded; one that gave up is VMB_ERR_TIMEOUT in
 *   vmb_read_status.
 * vmb_linear_bwd - given dy [M, N] bf16: dZ = dy act'(pre) (rounded to bf16, the slope at z as pre holds it, rounded
 *   too; pre may be NULL without an activation), dx = dZ weight [M, K], dweight = dZ^T x [N, K] (bf16; either may be NULL), dbias [N] fp32 (or NULL) the
 *   sums of dZ before its rounding.
 */
size_t vmb_causal_conv_workspace_bytes(int B, int T, int64_t total, int packed, int C, int W, vmb_dtype dtype);
vmb_status vmb_causal_conv_fwd(const void* x, const float* weight, const float* bias, const int64_t* strides,
                               const void* initial_state, const int32_t* offsets, void* y, void* final_state, int B,
                               int T, int64_t total, int C, int W, vmb_act act, vmb_dtype dtype, cudaStream_t stream);
vmb_status vmb_causal_conv_bwd(const void* x, const float* weight, const float* bias, const int64_t* strides,
                               const void* initial_state, const int32_t* offsets, const void* dy,
                               const void* dfinal_state, void* dx, float* dweight, float* dbias, void* dinitial_state,
                               int B, int T, int64_t total, int C, int W, vmb_act act, vmb_dtype dtype,
                               void* workspace, size_t workspace_bytes, cudaStream_t stream);
vmb_status vmb_causal_conv_step(const void* x, const float* weight, const float* bias, const int64_t* strides,
                                void* state, const int32_t* slots, void* y, int B, int T, int C, int W, int pool,
                                vmb_act act, vmb_dtype dtype, cudaStream_t stream);

size_t vmb_token_scan_workspace_bytes(int B, int T, int64_t total, int packed, int D, int N, int grads, vmb_dtype dtype);
size_t vmb_token_scan_saved_bytes(int B, int T, int64_t total, int packed, int D, int N);
vmb_status vmb_token_scan_fwd(const void* x, const void* delta, const float* A, const void* Bm, const void* Cm,
                              const float* Dskip, const float* delta_bias, const void* z, const int64_t* strides,
                              const float* initial_state, const int32_t* offsets, void* y, float* final_state,
                              void* saved, int B, int T, int64_t total, int D, int N, unsigned flags, vmb_dtype dtype,
                              void* workspace, size_t workspace_bytes, cudaStream_t stream);
vmb_status vmb_token_scan_bwd(const void* x, const void* delta, const float* A, const void* Bm, const void* Cm,
                              const float* Dskip, const float* delta_bias, const void* z, const int64_t* strides,
                              const int32_t* offsets, const void* dy, const float* dfinal_state, const void* saved,
                              void* dx, void* ddelta, float* dA, void* dBm, void* dCm, float* dDskip,
                              float* ddelta_bias, void* dz, float* dinitial_state, int B, int T, int64_t total, int D,
                              int N, unsigned flags, vmb_dtype dtype, void* workspace, size_t workspace_bytes,
                              cudaStream_t stream);
vmb_status vmb_token_scan_step(const void* x, const void* delta, const float* A, const void* Bm, const void* Cm,
                               const float* Dskip, const float* delta_bias, const void* z, const int64_t* strides,
                               float* state, const int32_t* slots, void* y, int B, int T, int D, int N, int pool,
                               unsigned flags, vmb_dtype dtype, cudaStream_t stream);

size_t vmb_rms_norm_workspace_bytes(int64_t rows, int C, vmb_dtype dtype);
vmb_status vmb_rms_norm_fwd(const void* x, const void* residual, const float* weight, void* y, void* sum, float* scale,
                            float* rstd, int64_t rows, int C, float eps, vmb_dtype dtype, cudaStream_t stream);
vmb_status vmb_rms_norm_bwd(const void* x, const float* weight, const float* rstd, const void* dy, const void* dsum,
                            void* dx, float* dweight, int64_t rows, int C, vmb_dtype dtype, void* workspace,
                            size_t workspace_bytes, cudaStream_t stream);

size_t vmb_linear_workspace_bytes(int64_t M, int K, int N, int grads);
vmb_status vmb_linear_fwd(const void* x, int64_t x_stride, const void* weight, const float* x_scale,
                          const float* weight_scale, const float* bias, const void* residual, void* y, void* pre,
                          int64_t M, int K, int N, vmb_act act, void* workspace, size_t workspace_bytes,
                          cudaStream_t stream);
vmb_status vmb_linear_bwd(const void* x, int64_t x_stride, const void* weight, const void* pre, const void* dy, void* dx,
                          void* dweight, float* dbias, int64_t M, int K, int N, vmb_act act, void* workspace,
                          size_t workspace_bytes, cudaStream_t stream);

/*
 * vmb_read_status - synchronise `stream`, then return and clear the device
 * error word of `workspace` (VMB_OK, VMB_ERR_TIMEOUT or VMB_ERR_BOUNDS).  A
 * device-side error leaves the outputs of that call undefined but the CUDA
 * context usable.  Returns VMB_ERR_CUDA if the synchronisation fails.
 */
vmb_status vmb_read_status(void* workspace, cudaStream_t stream);

/* Static description of a status code (never NULL). */
const char* vmb_status_string(vmb_status status);

/* Library version: major*10000 + minor*100 + patch. */
int vmb_version(void);

#ifdef __cplusplus
}
#endif

#endif /* VMB_H */
