"""Python binding of libvmb (include/vmb.h): argument marshalling only.

Every function has the name of the C entry point it calls and takes torch
CUDA tensors; it checks shapes and dtypes, allocates outputs with torch when
none are given, and passes raw device pointers plus the current CUDA stream
to the library.  All arithmetic runs in the library's kernels: there is no
fallback, and a missing library raises at import.
"""
from __future__ import annotations

import ctypes
import functools
import os
import threading

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libvmb.so")

VMB_OK = 0
VMB_ERR_INVALID_ARG = 1
VMB_ERR_MISALIGNED = 2
VMB_ERR_UNSUPPORTED = 3
VMB_ERR_WORKSPACE = 4
VMB_ERR_CUDA = 5
VMB_ERR_TIMEOUT = 6
VMB_ERR_BOUNDS = 7

VMB_F32 = 0
VMB_BF16 = 1

VMB_FLAG_SOFTPLUS = 0x1
VMB_FLAG_B_ZOH = 0x2
VMB_FLAG_SKIP_MEAN = 0x4
VMB_FLAG_TEST_SUPPRESS_PUBLISH = 0x40000000

VMB_PATH_FULL = 0
VMB_PATH_MEAN = 1

EXPORTS = ["vmb_cross_scan", "vmb_cross_merge", "vmb_scan_workspace_bytes", "vmb_scan_kernel_count",
           "vmb_selective_scan_fwd",
           "vmb_mean_scan_fwd", "vmb_mean_scan_merge_fwd", "vmb_mean_scan_grouped_fwd", "vmb_ss2d_mean_fwd",
           "vmb_ss2d_full_fwd", "vmb_discretise_fwd", "vmb_discretise_mean_fwd",
           "vmb_scan_only_fwd", "vmb_selection_fwd", "vmb_selection_lowrank_fwd", "vmb_selective_scan_lowrank_fwd",
           "vmb_mean_scan_lowrank_fwd", "vmb_mean_scan_train_fwd", "vmb_mean_scan_bwd",
           "vmb_mean_scan_bwd_workspace_bytes",
           "vmb_delta_rule_fwd", "vmb_delta_rule_bwd", "vmb_delta_rule_step", "vmb_delta_rule_workspace_bytes",
           "vmb_delta_rule_saved_bytes", "vmb_rotary_fwd", "vmb_group_norm_fwd", "vmb_group_norm_bwd",
           "vmb_group_norm_workspace_bytes",
           "vmb_causal_conv_fwd", "vmb_causal_conv_bwd", "vmb_causal_conv_step", "vmb_causal_conv_workspace_bytes",
           "vmb_token_scan_fwd", "vmb_token_scan_bwd", "vmb_token_scan_step", "vmb_token_scan_workspace_bytes",
           "vmb_token_scan_saved_bytes", "vmb_rms_norm_fwd", "vmb_rms_norm_bwd", "vmb_rms_norm_workspace_bytes",
           "vmb_linear_fwd", "vmb_linear_bwd", "vmb_linear_workspace_bytes",
           "vmb_read_status", "vmb_status_string", "vmb_version"]


class VmbError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status})")


def _load() -> ctypes.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built: run `python -c \"import __graft_entry__ as g; g.build()\"`")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i, u, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_uint, ctypes.c_size_t
    lib.vmb_cross_scan.argtypes = [vp, vp, i, i, i, i, i, vp]
    lib.vmb_cross_merge.argtypes = [vp, vp, i, i, i, i, i, vp]
    lib.vmb_scan_workspace_bytes.argtypes = [i, i, i, i, i, i, i, i]
    lib.vmb_scan_workspace_bytes.restype = sz
    lib.vmb_scan_kernel_count.argtypes = [i, i, i, i, i, i, i, i]
    lib.vmb_scan_kernel_count.restype = i
    lib.vmb_selective_scan_fwd.argtypes = [vp] * 8 + [i] * 6 + [u, i, vp, sz, vp]
    lib.vmb_mean_scan_fwd.argtypes = [vp] * 9 + [i] * 6 + [u, i, vp, sz, vp]
    lib.vmb_mean_scan_merge_fwd.argtypes = [vp] * 10 + [i] * 5 + [u, i, vp, sz, vp]
    lib.vmb_ss2d_mean_fwd.argtypes = [vp] * 10 + [i] * 5 + [u, i, vp, sz, vp]
    lib.vmb_ss2d_full_fwd.argtypes = [vp] * 10 + [i] * 5 + [u, i, vp, sz, vp]
    lib.vmb_mean_scan_grouped_fwd.argtypes = [vp] * 9 + [i] * 7 + [u, i, vp, sz, vp]
    lib.vmb_discretise_fwd.argtypes = [vp] * 7 + [i] * 6 + [u, i, vp]
    lib.vmb_discretise_mean_fwd.argtypes = [vp] * 7 + [i] * 6 + [u, i, vp]
    lib.vmb_scan_only_fwd.argtypes = [vp] * 4 + [i] * 6 + [i, vp]
    lib.vmb_selection_fwd.argtypes = [vp] * 8 + [i] * 7 + [i, vp]
    lib.vmb_selection_lowrank_fwd.argtypes = [vp] * 7 + [i] * 7 + [i, vp]
    lib.vmb_selective_scan_lowrank_fwd.argtypes = [vp] * 9 + [i] * 7 + [u, i, vp, sz, vp]
    lib.vmb_mean_scan_lowrank_fwd.argtypes = [vp] * 10 + [i] * 7 + [u, i, vp, sz, vp]
    lib.vmb_mean_scan_train_fwd.argtypes = [vp] * 10 + [i] * 7 + [u, i, vp, sz, vp]
    lib.vmb_mean_scan_bwd.argtypes = [vp] * 16 + [i] * 7 + [u, i, vp, sz, vp]
    lib.vmb_mean_scan_bwd_workspace_bytes.argtypes = [i] * 8
    lib.vmb_mean_scan_bwd_workspace_bytes.restype = sz
    f, i64 = ctypes.c_float, ctypes.c_int64
    lib.vmb_delta_rule_fwd.argtypes = [vp] * 11 + [i, i, i64, i, i, i, i, f, i, vp, sz, vp]
    lib.vmb_delta_rule_bwd.argtypes = [vp] * 15 + [i, i, i64, i, i, i, i, f, i, vp, sz, vp]
    lib.vmb_delta_rule_step.argtypes = [vp] * 9 + [i] * 7 + [f, i, vp]
    lib.vmb_delta_rule_workspace_bytes.argtypes = [i, i, i64, i, i, i, i, i, i, i]
    lib.vmb_delta_rule_workspace_bytes.restype = sz
    lib.vmb_delta_rule_saved_bytes.argtypes = [i, i, i64, i, i, i, i, i]
    lib.vmb_delta_rule_saved_bytes.restype = sz
    lib.vmb_rotary_fwd.argtypes = [vp] * 6 + [i] * 6 + [vp, vp, vp, u, i, vp]
    lib.vmb_group_norm_fwd.argtypes = [vp] * 5 + [i, i64, i, i, f, i, i, vp, sz, vp]
    lib.vmb_group_norm_bwd.argtypes = [vp] * 8 + [i, i64, i, i, i, i, vp, sz, vp]
    lib.vmb_group_norm_workspace_bytes.argtypes = [i, i64, i, i, i, i]
    lib.vmb_group_norm_workspace_bytes.restype = sz
    lib.vmb_causal_conv_fwd.argtypes = [vp] * 8 + [i, i, i64, i, i, i, i, vp]
    lib.vmb_causal_conv_bwd.argtypes = [vp] * 12 + [i, i, i64, i, i, i, i, vp, sz, vp]
    lib.vmb_causal_conv_step.argtypes = [vp] * 7 + [i] * 7 + [vp]
    lib.vmb_causal_conv_workspace_bytes.argtypes = [i, i, i64, i, i, i, i]
    lib.vmb_token_scan_fwd.argtypes = [vp] * 14 + [i, i, i64, i, i, u, i, vp, sz, vp]
    lib.vmb_token_scan_bwd.argtypes = [vp] * 22 + [i, i, i64, i, i, u, i, vp, sz, vp]
    lib.vmb_token_scan_step.argtypes = [vp] * 12 + [i] * 5 + [u, i, vp]
    lib.vmb_token_scan_workspace_bytes.argtypes = [i, i, i64, i, i, i, i, i]
    lib.vmb_token_scan_saved_bytes.argtypes = [i, i, i64, i, i, i]
    lib.vmb_rms_norm_fwd.argtypes = [vp] * 7 + [i64, i, f, i, vp]
    lib.vmb_rms_norm_bwd.argtypes = [vp] * 7 + [i64, i, i, vp, sz, vp]
    lib.vmb_rms_norm_workspace_bytes.argtypes = [i64, i, i]
    lib.vmb_linear_fwd.argtypes = [vp, i64] + [vp] * 7 + [i64, i, i, i, vp, sz, vp]
    lib.vmb_linear_bwd.argtypes = [vp, i64] + [vp] * 6 + [i64, i, i, i, vp, sz, vp]
    lib.vmb_linear_workspace_bytes.argtypes = [i64, i, i, i]
    for name in ["vmb_causal_conv_workspace_bytes", "vmb_token_scan_workspace_bytes", "vmb_token_scan_saved_bytes",
                 "vmb_rms_norm_workspace_bytes", "vmb_linear_workspace_bytes"]:
        getattr(lib, name).restype = sz
    lib.vmb_read_status.argtypes = [vp, vp]
    lib.vmb_status_string.argtypes = [i]
    lib.vmb_status_string.restype = ctypes.c_char_p
    lib.vmb_version.argtypes = []
    for name in ["vmb_cross_scan", "vmb_cross_merge", "vmb_selective_scan_fwd", "vmb_mean_scan_fwd",
                 "vmb_mean_scan_merge_fwd", "vmb_mean_scan_grouped_fwd", "vmb_ss2d_mean_fwd", "vmb_ss2d_full_fwd",
                 "vmb_discretise_fwd",
                 "vmb_discretise_mean_fwd", "vmb_scan_only_fwd", "vmb_selection_fwd", "vmb_mean_scan_bwd",
                 "vmb_selection_lowrank_fwd", "vmb_selective_scan_lowrank_fwd", "vmb_mean_scan_lowrank_fwd",
                 "vmb_delta_rule_fwd", "vmb_delta_rule_bwd", "vmb_delta_rule_step", "vmb_rotary_fwd",
                 "vmb_group_norm_fwd", "vmb_group_norm_bwd",
                 "vmb_causal_conv_fwd", "vmb_causal_conv_bwd", "vmb_causal_conv_step", "vmb_token_scan_fwd",
                 "vmb_token_scan_bwd", "vmb_token_scan_step", "vmb_rms_norm_fwd", "vmb_rms_norm_bwd",
                 "vmb_linear_fwd", "vmb_linear_bwd",
                 "vmb_read_status", "vmb_version"]:
        getattr(lib, name).restype = i
    return lib


lib = _load()


def status_string(status: int) -> str:
    return lib.vmb_status_string(int(status)).decode()


def vmb_status_string(status: int) -> str:
    return status_string(status)


def vmb_version() -> int:
    return lib.vmb_version()


def _check(status: int, where: str):
    if status != VMB_OK:
        raise VmbError(status, where)


def _dtype_code(t: torch.dtype) -> int:
    if t == torch.float32:
        return VMB_F32
    if t == torch.bfloat16:
        return VMB_BF16
    raise TypeError(f"unsupported dtype {t} (float32 or bfloat16)")


def _ptr(t):
    return t.data_ptr() if t is not None else None


def _dev(t: torch.Tensor, name: str):
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t


def _stream(stream) -> int:
    s = torch.cuda.current_stream() if stream is None else stream
    return s.cuda_stream


_raw_stream = torch._C._cuda_getCurrentRawStream
_current_device = torch._C._cuda_getDevice


@functools.lru_cache(maxsize=None)
def _several_devices() -> bool:
    return torch.cuda.device_count() > 1


def _on_its_stream(call):
    """`call` on the device of its first tensor and with `stream` as the current stream: what it allocates and fills belongs
    to the stream that it launches on."""
    @functools.wraps(call)
    def wrapped(*args, stream=None, **kwargs):
        if stream is None and not _several_devices():
            return call(*args, **kwargs)
        index = next((t.get_device() for t in (*args, *kwargs.values()) if isinstance(t, torch.Tensor)), -1)
        if index >= 0 and stream is not None and stream.device_index != index:
            raise ValueError("the stream belongs to another device than the tensors")
        if index >= 0 and index != _current_device():
            with torch.cuda.device(index):
                return wrapped(*args, stream=stream, **kwargs)
        if stream is None:
            return call(*args, **kwargs)
        with torch.cuda.stream(stream):
            return call(*args, stream=stream, **kwargs)
    return wrapped


def _one_device(first, *others):
    """All of these CUDA tensors (or None) are on one device."""
    if _several_devices():
        index = first.get_device()
        for t in others:
            if t is not None and t.get_device() != index:
                raise ValueError("all tensors of a call must be on one device")


# ---------------------------------------------------------------- cross-scan / merge


@_on_its_stream
def vmb_cross_scan(x: torch.Tensor, xs: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """x [B, D, H, W] -> xs [B, 4, D, H*W] (bit-exact permutation)."""
    _dev(x, "x")
    B, D, H, W = x.shape
    if xs is None:
        xs = torch.empty((B, 4, D, H * W), dtype=x.dtype, device=x.device)
    _dev(xs, "xs")
    if xs.shape != (B, 4, D, H * W) or xs.dtype != x.dtype:
        raise ValueError("xs must be [B, 4, D, H*W] with the dtype of x")
    _check(lib.vmb_cross_scan(_ptr(x), _ptr(xs), B, D, H, W, _dtype_code(x.dtype), _stream(stream)),
           "vmb_cross_scan")
    return xs


@_on_its_stream
def vmb_cross_merge(ys: torch.Tensor, H: int, W: int, out: torch.Tensor | None = None,
                    stream=None) -> torch.Tensor:
    """ys [B, 4, D, H*W] -> out [B, D, H, W]."""
    _dev(ys, "ys")
    B, K, D, L = ys.shape
    if K != 4 or L != H * W:
        raise ValueError("ys must be [B, 4, D, H*W]")
    if out is None:
        out = torch.empty((B, D, H, W), dtype=ys.dtype, device=ys.device)
    _dev(out, "out")
    if out.shape != (B, D, H, W) or out.dtype != ys.dtype:
        raise ValueError("out must be [B, D, H, W] with the dtype of ys")
    _check(lib.vmb_cross_merge(_ptr(ys), _ptr(out), B, D, H, W, _dtype_code(ys.dtype), _stream(stream)),
           "vmb_cross_merge")
    return out


# ---------------------------------------------------------------- scans


def vmb_scan_workspace_bytes(path: int, B: int, K: int, D: int, N: int, H: int, W: int,
                             dtype: torch.dtype = torch.float32) -> int:
    return int(lib.vmb_scan_workspace_bytes(path, B, K, D, N, H, W, _dtype_code(dtype)))


def vmb_scan_kernel_count(path: int, B: int, K: int, D: int, N: int, H: int, W: int,
                          dtype: torch.dtype = torch.float32) -> int:
    return int(lib.vmb_scan_kernel_count(path, B, K, D, N, H, W, _dtype_code(dtype)))


class Workspace:
    """Zero-initialised device workspaces that grow on demand: one per thread, device and current stream, so that calls
    which may overlap in time never share one.

    A buffer is allocated and zero-filled on the stream whose calls use it, which also orders the reuse of the memory of
    a buffer that was outgrown.  The library keeps a workspace ready for the next call by itself.  While the stream is
    being captured into a graph every call gets a buffer of its own, which the graph fills and holds: a kept one would be
    shared by the graph's replays and later calls, and one made during the capture is not filled before a replay."""

    def __init__(self, header: int = 0):
        """`header`: the bytes that have to be zero at first; 0: all."""
        self._local = threading.local()
        self._header = header

    def buffers(self) -> dict:
        """(device index, raw stream) -> buffer, of the calling thread."""
        try:
            return self._local.bufs
        except AttributeError:
            self._local.bufs = {}
            return self._local.bufs

    def outgrown(self) -> dict:
        """The same of the calling thread's buffers that were outgrown: their headers, for the errors that nobody has read."""
        try:
            return self._local.left
        except AttributeError:
            self._local.left = {}
            return self._local.left

    def get(self, nbytes: int, device: torch.device) -> torch.Tensor:
        index = torch.cuda.current_device() if device.index is None else device.index
        bufs, key = self.buffers(), (index, _raw_stream(index))
        capturing = torch.cuda.is_current_stream_capturing()
        buf = bufs.get(key)
        if buf is None or buf.numel() < nbytes or capturing:
            n = (max(nbytes, 256) + 255) // 256 * 256
            device = torch.device("cuda", index)
            if self._header:  # (a call captured into a graph gets a buffer of its own: the rest is not filled at every replay)
                buf = torch.empty(n, dtype=torch.uint8, device=device)
                buf[:self._header].zero_()
            else:
                buf = torch.zeros(n, dtype=torch.uint8, device=device)
            if not capturing:
                old, left = bufs.get(key), self.outgrown()
                if old is not None:
                    left[key] = left[key] | old[:256] if key in left else old[:256].clone()
                bufs[key] = buf
        return buf


_default_ws = Workspace()


def _scan_shapes(u, delta, A, Bs, Cs, Dskip, delta_bias, H, W):
    for t, n in [(u, "u"), (delta, "delta"), (A, "A"), (Bs, "Bs"), (Cs, "Cs"), (Dskip, "Dskip"),
                 (delta_bias, "delta_bias")]:
        _dev(t, n)
    B, K, D, L = u.shape
    N = Bs.shape[2]
    if L != H * W:
        raise ValueError("u must be [B, K, D, H*W]")
    if delta.shape != u.shape or Bs.shape != (B, K, N, L) or Cs.shape != (B, K, N, L):
        raise ValueError("delta [B,K,D,L], Bs and Cs [B,K,N,L] expected")
    if len({u.dtype, delta.dtype, Bs.dtype, Cs.dtype}) != 1:
        raise ValueError("u, delta, Bs, Cs must share one dtype")
    if A.shape != (K * D, N) or Dskip.shape != (K * D,) or delta_bias.shape != (K * D,):
        raise ValueError("A [K*D, N], Dskip [K*D], delta_bias [K*D] expected")
    if A.dtype != torch.float32 or Dskip.dtype != torch.float32 or delta_bias.dtype != torch.float32:
        raise ValueError("A, Dskip, delta_bias must be float32")
    return B, K, D, N, L


@_on_its_stream
def vmb_selective_scan_fwd(u, delta, A, Bs, Cs, Dskip, delta_bias, H: int, W: int, *,
                           y=None, flags: int = VMB_FLAG_SOFTPLUS, workspace=None,
                           stream=None) -> torch.Tensor:
    """Full-channel selective scan: y [B, K, D, H*W] (dtype of u)."""
    B, K, D, N, L = _scan_shapes(u, delta, A, Bs, Cs, Dskip, delta_bias, H, W)
    if y is None:
        y = torch.empty_like(u)
    _dev(y, "y")
    if y.shape != u.shape or y.dtype != u.dtype:
        raise ValueError("y must match u")
    ws_bytes = vmb_scan_workspace_bytes(VMB_PATH_FULL, B, K, D, N, H, W, u.dtype)
    if workspace is None:
        workspace = _default_ws.get(ws_bytes, u.device)
    _check(lib.vmb_selective_scan_fwd(_ptr(u), _ptr(delta), _ptr(A), _ptr(Bs), _ptr(Cs), _ptr(Dskip),
                                      _ptr(delta_bias), _ptr(y), B, K, D, N, H, W, flags,
                                      _dtype_code(u.dtype), _ptr(workspace), workspace.numel(),
                                      _stream(stream)), "vmb_selective_scan_fwd")
    return y


@_on_its_stream
def vmb_mean_scan_fwd(u, delta, A, Bs, Cs, Dskip, delta_bias, H: int, W: int, *,
                      y=None, ybar=None, want_ybar: bool = False, flags: int = VMB_FLAG_SOFTPLUS,
                      workspace=None, stream=None):
    """VMeanba channel-mean scan: returns (y [B, K, D, L], ybar [B, K, L] fp32 or None)."""
    B, K, D, N, L = _scan_shapes(u, delta, A, Bs, Cs, Dskip, delta_bias, H, W)
    if y is None:
        y = torch.empty_like(u)
    _dev(y, "y")
    if y.shape != u.shape or y.dtype != u.dtype:
        raise ValueError("y must match u")
    if ybar is None and want_ybar:
        ybar = torch.empty((B, K, L), dtype=torch.float32, device=u.device)
    if ybar is not None:
        _dev(ybar, "ybar")
        if ybar.shape != (B, K, L) or ybar.dtype != torch.float32:
            raise ValueError("ybar must be float32 [B, K, L]")
    ws_bytes = vmb_scan_workspace_bytes(VMB_PATH_MEAN, B, K, D, N, H, W, u.dtype)
    if workspace is None:
        workspace = _default_ws.get(ws_bytes, u.device)
    _check(lib.vmb_mean_scan_fwd(_ptr(u), _ptr(delta), _ptr(A), _ptr(Bs), _ptr(Cs), _ptr(Dskip),
                                 _ptr(delta_bias), _ptr(y), _ptr(ybar), B, K, D, N, H, W, flags,
                                 _dtype_code(u.dtype), _ptr(workspace), workspace.numel(),
                                 _stream(stream)), "vmb_mean_scan_fwd")
    return y, ybar


@_on_its_stream
def vmb_mean_scan_grouped_fwd(u, delta, A, Bs, Cs, Dskip, delta_bias, H: int, W: int, groups: int, *,
                              y=None, ybar=None, want_ybar: bool = False, flags: int = VMB_FLAG_SOFTPLUS,
                              workspace=None, stream=None):
    """Grouped basis (reduced channel dimension d = groups): the channel mean of Eq. 9 over each
    of `groups` channel groups; returns (y [B, K, D, L], ybar [B, K, groups, L] fp32 or None)."""
    B, K, D, N, L = _scan_shapes(u, delta, A, Bs, Cs, Dskip, delta_bias, H, W)
    if groups < 1 or D % groups:
        raise ValueError("groups must be >= 1 and divide D")
    if y is None:
        y = torch.empty_like(u)
    _dev(y, "y")
    if y.shape != u.shape or y.dtype != u.dtype:
        raise ValueError("y must match u")
    if ybar is None and want_ybar:
        ybar = torch.empty((B, K, groups, L), dtype=torch.float32, device=u.device)
    if ybar is not None:
        _dev(ybar, "ybar")
        if ybar.shape != (B, K, groups, L) or ybar.dtype != torch.float32:
            raise ValueError("ybar must be float32 [B, K, groups, L]")
    ws_bytes = vmb_scan_workspace_bytes(VMB_PATH_MEAN, B, K * groups, D // groups, N, H, W, u.dtype)
    if workspace is None:
        workspace = _default_ws.get(ws_bytes, u.device)
    _check(lib.vmb_mean_scan_grouped_fwd(_ptr(u), _ptr(delta), _ptr(A), _ptr(Bs), _ptr(Cs), _ptr(Dskip),
                                         _ptr(delta_bias), _ptr(y), _ptr(ybar), B, K, D, N, H, W, groups, flags,
                                         _dtype_code(u.dtype), _ptr(workspace), workspace.numel(),
                                         _stream(stream)), "vmb_mean_scan_grouped_fwd")
    return y, ybar


@_on_its_stream
def vmb_mean_scan_train_fwd(u, delta, A, Bs, Cs, Dskip, delta_bias, H: int, W: int, *, groups: int = 1,
                            y=None, ybar=None, saved=None, flags: int = VMB_FLAG_SOFTPLUS, workspace=None,
                            stream=None):
    """The (grouped) channel-mean scan that also keeps its group means for the backward: returns
    (y [B, K, D, L], saved [B, K, groups, N + 1, L] fp32, ybar or None)."""
    B, K, D, N, L = _scan_shapes(u, delta, A, Bs, Cs, Dskip, delta_bias, H, W)
    if groups < 1 or D % groups:
        raise ValueError("groups must be >= 1 and divide D")
    if y is None:
        y = torch.empty_like(u)
    _dev(y, "y")
    if y.shape != u.shape or y.dtype != u.dtype:
        raise ValueError("y must match u")
    if saved is None:
        saved = torch.empty((B, K, groups, N + 1, L), dtype=torch.float32, device=u.device)
    _dev(saved, "saved")
    if tuple(saved.shape) != (B, K, groups, N + 1, L) or saved.dtype != torch.float32:
        raise ValueError("saved must be float32 [B, K, groups, N + 1, L]")
    if ybar is not None:
        _dev(ybar, "ybar")
        if ybar.shape != (B, K, groups, L) or ybar.dtype != torch.float32:
            raise ValueError("ybar must be float32 [B, K, groups, L]")
    ws_bytes = vmb_scan_workspace_bytes(VMB_PATH_MEAN, B, K * groups, D // groups, N, H, W, u.dtype)
    if workspace is None:
        workspace = _default_ws.get(ws_bytes, u.device)
    _check(lib.vmb_mean_scan_train_fwd(_ptr(u), _ptr(delta), _ptr(A), _ptr(Bs), _ptr(Cs), _ptr(Dskip),
                                       _ptr(delta_bias), _ptr(y), _ptr(ybar), _ptr(saved), B, K, D, N, H, W, groups,
                                       flags, _dtype_code(u.dtype), _ptr(workspace), workspace.numel(),
                                       _stream(stream)), "vmb_mean_scan_train_fwd")
    return y, saved, ybar


@_on_its_stream
def vmb_mean_scan_merge_fwd(u, delta, A, Bs, Cs, Dskip, delta_bias, x, H: int, W: int, *,
                            out=None, ybar=None, flags: int = VMB_FLAG_SOFTPLUS, workspace=None, stream=None):
    """Channel-mean path with the broadcast fused into the cross-merge:
    returns (out [B, D, H, W], ybar [B, 4, L] fp32)."""
    B, K, D, N, L = _scan_shapes(u, delta, A, Bs, Cs, Dskip, delta_bias, H, W)
    if K != 4:
        raise ValueError("the fused merge needs the four SS2D directions (K = 4)")
    _dev(x, "x")
    if tuple(x.shape) != (B, D, H, W) or x.dtype != u.dtype:
        raise ValueError("x must be [B, D, H, W] in the storage dtype of u")
    if out is None:
        out = torch.empty_like(x)
    _dev(out, "out")
    if out.shape != x.shape or out.dtype != x.dtype:
        raise ValueError("out must match x")
    if ybar is None:
        ybar = torch.empty((B, 4, L), dtype=torch.float32, device=u.device)
    _dev(ybar, "ybar")
    if ybar.shape != (B, 4, L) or ybar.dtype != torch.float32:
        raise ValueError("ybar must be float32 [B, 4, L]")
    ws_bytes = vmb_scan_workspace_bytes(VMB_PATH_MEAN, B, 4, D, N, H, W, u.dtype)
    if workspace is None:
        workspace = _default_ws.get(ws_bytes, u.device)
    _check(lib.vmb_mean_scan_merge_fwd(_ptr(u), _ptr(delta), _ptr(A), _ptr(Bs), _ptr(Cs), _ptr(Dskip),
                                       _ptr(delta_bias), _ptr(x), _ptr(out), _ptr(ybar), B, D, N, H, W, flags,
                                       _dtype_code(u.dtype), _ptr(workspace), workspace.numel(),
                                       _stream(stream)), "vmb_mean_scan_merge_fwd")
    return out, ybar


@_on_its_stream
def vmb_ss2d_mean_fwd(x, delta, A, Bs, Cs, Dskip, delta_bias, *, out=None, ybar=None, xt=None,
                      flags: int = VMB_FLAG_SOFTPLUS, workspace=None, stream=None):
    """The scan side of a VMeanba SS2D block from the map: cross-scan, channel-mean scan and
    cross-merge in one call, xs and y never written.  x [B, D, H, W]; delta [B, 4, D, H*W],
    Bs, Cs [B, 4, N, H*W]; xt [B, D, W, H] scratch for the map's transpose (allocated when not
    given); returns (out [B, D, H, W], ybar [B, 4, H*W] fp32)."""
    _dev(x, "x")
    B, D, H, W = x.shape
    if xt is None:
        xt = torch.empty((B, D, W, H), dtype=x.dtype, device=x.device)
    _dev(xt, "xt")
    if tuple(xt.shape) != (B, D, W, H) or xt.dtype != x.dtype:
        raise ValueError("xt must be [B, D, W, H] in the dtype of x")
    L = H * W
    for t, n in [(delta, "delta"), (A, "A"), (Bs, "Bs"), (Cs, "Cs"), (Dskip, "Dskip"), (delta_bias, "delta_bias")]:
        _dev(t, n)
    N = Bs.shape[2]
    if tuple(delta.shape) != (B, 4, D, L) or tuple(Bs.shape) != (B, 4, N, L) or tuple(Cs.shape) != (B, 4, N, L):
        raise ValueError("delta [B,4,D,H*W], Bs and Cs [B,4,N,H*W] expected")
    if len({x.dtype, delta.dtype, Bs.dtype, Cs.dtype}) != 1:
        raise ValueError("x, delta, Bs, Cs must share one dtype")
    if tuple(A.shape) != (4 * D, N) or tuple(Dskip.shape) != (4 * D,) or tuple(delta_bias.shape) != (4 * D,):
        raise ValueError("A [4*D, N], Dskip [4*D], delta_bias [4*D] expected")
    if A.dtype != torch.float32 or Dskip.dtype != torch.float32 or delta_bias.dtype != torch.float32:
        raise ValueError("A, Dskip, delta_bias must be float32")
    if out is None:
        out = torch.empty_like(x)
    _dev(out, "out")
    if out.shape != x.shape or out.dtype != x.dtype:
        raise ValueError("out must match x")
    if ybar is None:
        ybar = torch.empty((B, 4, L), dtype=torch.float32, device=x.device)
    _dev(ybar, "ybar")
    if tuple(ybar.shape) != (B, 4, L) or ybar.dtype != torch.float32:
        raise ValueError("ybar must be float32 [B, 4, L]")
    ws_bytes = vmb_scan_workspace_bytes(VMB_PATH_MEAN, B, 4, D, N, H, W, x.dtype)
    if workspace is None:
        workspace = _default_ws.get(ws_bytes, x.device)
    _check(lib.vmb_ss2d_mean_fwd(_ptr(x), _ptr(xt), _ptr(delta), _ptr(A), _ptr(Bs), _ptr(Cs), _ptr(Dskip),
                                 _ptr(delta_bias),
                                 _ptr(out), _ptr(ybar), B, D, N, H, W, flags, _dtype_code(x.dtype), _ptr(workspace),
                                 workspace.numel(), _stream(stream)), "vmb_ss2d_mean_fwd")
    return out, ybar


@_on_its_stream
def vmb_ss2d_full_fwd(x, delta, A, Bs, Cs, Dskip, delta_bias, *, out=None, y=None, xt=None,
                      flags: int = VMB_FLAG_SOFTPLUS, workspace=None, stream=None):
    """The scan side of a full-channel SS2D block from the map: cross-scan, selective scan and
    cross-merge in one call, xs never written.  x [B, D, H, W]; delta [B, 4, D, H*W], Bs, Cs
    [B, 4, N, H*W]; xt [B, D, W, H] scratch for the map's transpose (allocated when not given);
    returns (out [B, D, H, W], y [B, 4, D, H*W])."""
    _dev(x, "x")
    B, D, H, W = x.shape
    if xt is None:
        xt = torch.empty((B, D, W, H), dtype=x.dtype, device=x.device)
    _dev(xt, "xt")
    if tuple(xt.shape) != (B, D, W, H) or xt.dtype != x.dtype:
        raise ValueError("xt must be [B, D, W, H] in the dtype of x")
    L = H * W
    for t, n in [(delta, "delta"), (A, "A"), (Bs, "Bs"), (Cs, "Cs"), (Dskip, "Dskip"), (delta_bias, "delta_bias")]:
        _dev(t, n)
    N = Bs.shape[2]
    if tuple(delta.shape) != (B, 4, D, L) or tuple(Bs.shape) != (B, 4, N, L) or tuple(Cs.shape) != (B, 4, N, L):
        raise ValueError("delta [B,4,D,H*W], Bs and Cs [B,4,N,H*W] expected")
    if len({x.dtype, delta.dtype, Bs.dtype, Cs.dtype}) != 1:
        raise ValueError("x, delta, Bs, Cs must share one dtype")
    if tuple(A.shape) != (4 * D, N) or tuple(Dskip.shape) != (4 * D,) or tuple(delta_bias.shape) != (4 * D,):
        raise ValueError("A [4*D, N], Dskip [4*D], delta_bias [4*D] expected")
    if A.dtype != torch.float32 or Dskip.dtype != torch.float32 or delta_bias.dtype != torch.float32:
        raise ValueError("A, Dskip, delta_bias must be float32")
    if out is None:
        out = torch.empty_like(x)
    _dev(out, "out")
    if out.shape != x.shape or out.dtype != x.dtype:
        raise ValueError("out must match x")
    if y is None:
        y = torch.empty((B, 4, D, L), dtype=x.dtype, device=x.device)
    _dev(y, "y")
    if tuple(y.shape) != (B, 4, D, L) or y.dtype != x.dtype:
        raise ValueError("y must be [B, 4, D, H*W] in the dtype of x")
    ws_bytes = vmb_scan_workspace_bytes(VMB_PATH_FULL, B, 4, D, N, H, W, x.dtype)
    if workspace is None:
        workspace = _default_ws.get(ws_bytes, x.device)
    _check(lib.vmb_ss2d_full_fwd(_ptr(x), _ptr(xt), _ptr(delta), _ptr(A), _ptr(Bs), _ptr(Cs), _ptr(Dskip),
                                 _ptr(delta_bias), _ptr(y), _ptr(out), B, D, N, H, W, flags, _dtype_code(x.dtype),
                                 _ptr(workspace), workspace.numel(), _stream(stream)), "vmb_ss2d_full_fwd")
    return out, y


# ------------------------------------------- the paper's scan-only kernel setting


def _disc_shapes(u, delta, A, Bs, delta_bias, H, W):
    for t, n in [(u, "u"), (delta, "delta"), (A, "A"), (Bs, "Bs"), (delta_bias, "delta_bias")]:
        _dev(t, n)
    B, K, D, L = u.shape
    N = Bs.shape[2]
    if L != H * W or delta.shape != u.shape or Bs.shape != (B, K, N, L):
        raise ValueError("u, delta [B,K,D,H*W] and Bs [B,K,N,H*W] expected")
    if len({u.dtype, delta.dtype, Bs.dtype}) != 1:
        raise ValueError("u, delta, Bs must share one dtype")
    if A.shape != (K * D, N) or delta_bias.shape != (K * D,) or A.dtype != torch.float32 \
            or delta_bias.dtype != torch.float32:
        raise ValueError("A [K*D, N], delta_bias [K*D] float32 expected")
    return B, K, D, N, L


@_on_its_stream
def vmb_discretise_fwd(u, delta, A, Bs, delta_bias, H: int, W: int, *, dA=None, dBu=None,
                       flags: int = VMB_FLAG_SOFTPLUS, stream=None):
    """Eqs. 4, 6 outside the scan: (dA, dBu), each float32 [B, K, D, N, H*W]."""
    B, K, D, N, L = _disc_shapes(u, delta, A, Bs, delta_bias, H, W)
    shape = (B, K, D, N, L)
    dA = torch.empty(shape, dtype=torch.float32, device=u.device) if dA is None else dA
    dBu = torch.empty(shape, dtype=torch.float32, device=u.device) if dBu is None else dBu
    for t, n in [(dA, "dA"), (dBu, "dBu")]:
        _dev(t, n)
        if t.shape != shape or t.dtype != torch.float32:
            raise ValueError(f"{n} must be float32 {shape}")
    _check(lib.vmb_discretise_fwd(_ptr(u), _ptr(delta), _ptr(A), _ptr(Bs), _ptr(delta_bias), _ptr(dA), _ptr(dBu),
                                  B, K, D, N, H, W, flags, _dtype_code(u.dtype), _stream(stream)),
           "vmb_discretise_fwd")
    return dA, dBu


@_on_its_stream
def vmb_discretise_mean_fwd(u, delta, A, Bs, delta_bias, H: int, W: int, *, dAm=None, dBum=None,
                            flags: int = VMB_FLAG_SOFTPLUS, stream=None):
    """Channel means of the discretised operands (Eq. 9's T): (dAm, dBum), float32 [B, K, N, H*W]."""
    B, K, D, N, L = _disc_shapes(u, delta, A, Bs, delta_bias, H, W)
    shape = (B, K, N, L)
    dAm = torch.empty(shape, dtype=torch.float32, device=u.device) if dAm is None else dAm
    dBum = torch.empty(shape, dtype=torch.float32, device=u.device) if dBum is None else dBum
    for t, n in [(dAm, "dAm"), (dBum, "dBum")]:
        _dev(t, n)
        if t.shape != shape or t.dtype != torch.float32:
            raise ValueError(f"{n} must be float32 {shape}")
    _check(lib.vmb_discretise_mean_fwd(_ptr(u), _ptr(delta), _ptr(A), _ptr(Bs), _ptr(delta_bias), _ptr(dAm),
                                       _ptr(dBum), B, K, D, N, H, W, flags, _dtype_code(u.dtype), _stream(stream)),
           "vmb_discretise_mean_fwd")
    return dAm, dBum


@_on_its_stream
def vmb_scan_only_fwd(dA, dBu, Cs, H: int, W: int, *, y=None, stream=None):
    """The scan alone (Eq. 3 without the skip): dA, dBu float32 [B, K, Dm, N, L] (or
    [B, K, N, L] for one channel), Cs [B, K, N, L] -> y float32 [B, K, Dm, L] (or [B, K, L])."""
    for t, n in [(dA, "dA"), (dBu, "dBu"), (Cs, "Cs")]:
        _dev(t, n)
    one = dA.dim() == 4
    B, K = dA.shape[:2]
    Dm = 1 if one else dA.shape[2]
    N, L = dA.shape[-2:]
    if L != H * W or dBu.shape != dA.shape or Cs.shape != (B, K, N, L):
        raise ValueError("dA, dBu [B,K,Dm,N,H*W] and Cs [B,K,N,H*W] expected")
    if dA.dtype != torch.float32 or dBu.dtype != torch.float32:
        raise ValueError("dA, dBu must be float32")
    shape = (B, K, L) if one else (B, K, Dm, L)
    y = torch.empty(shape, dtype=torch.float32, device=dA.device) if y is None else y
    _dev(y, "y")
    if tuple(y.shape) != shape or y.dtype != torch.float32:
        raise ValueError(f"y must be float32 {shape}")
    _check(lib.vmb_scan_only_fwd(_ptr(dA), _ptr(dBu), _ptr(Cs), _ptr(y), B, K, Dm, N, H, W, _dtype_code(Cs.dtype),
                                 _stream(stream)), "vmb_scan_only_fwd")
    return y


@_on_its_stream
def vmb_selection_fwd(u, WB, WC, Wz, Wup, H: int, W: int, *, delta_raw=None, Bs=None, Cs=None, stream=None):
    """Eq. 6 selection functions: u [B, K, D, H*W] -> (delta_raw [B, K, D, L], Bs, Cs [B, K, N, L]),
    all in u's dtype; WB, WC [K, N, D], Wz [K, R, D], Wup [K, D, R] float32."""
    for t, n in [(u, "u"), (WB, "WB"), (WC, "WC"), (Wz, "Wz"), (Wup, "Wup")]:
        _dev(t, n)
    B, K, D, L = u.shape
    N, R = WB.shape[1], Wz.shape[1]
    if L != H * W or tuple(WB.shape) != (K, N, D) or tuple(WC.shape) != (K, N, D) or \
            tuple(Wz.shape) != (K, R, D) or tuple(Wup.shape) != (K, D, R):
        raise ValueError("u [B,K,D,H*W], WB/WC [K,N,D], Wz [K,R,D], Wup [K,D,R] expected")
    if any(w.dtype != torch.float32 for w in (WB, WC, Wz, Wup)):
        raise ValueError("weights must be float32")
    delta_raw = torch.empty_like(u) if delta_raw is None else delta_raw
    Bs = torch.empty((B, K, N, L), dtype=u.dtype, device=u.device) if Bs is None else Bs
    Cs = torch.empty((B, K, N, L), dtype=u.dtype, device=u.device) if Cs is None else Cs
    for t, n, shp in [(delta_raw, "delta_raw", (B, K, D, L)), (Bs, "Bs", (B, K, N, L)), (Cs, "Cs", (B, K, N, L))]:
        _dev(t, n)
        if tuple(t.shape) != shp or t.dtype != u.dtype:
            raise ValueError(f"{n} must be {u.dtype} {shp}")
    _check(lib.vmb_selection_fwd(_ptr(u), _ptr(WB), _ptr(WC), _ptr(Wz), _ptr(Wup), _ptr(Bs), _ptr(Cs),
                                 _ptr(delta_raw), B, K, D, N, R, H, W, _dtype_code(u.dtype), _stream(stream)),
           "vmb_selection_fwd")
    return delta_raw, Bs, Cs


@_on_its_stream
def vmb_selection_lowrank_fwd(u, WB, WC, Wz, H: int, W: int, *, z=None, Bs=None, Cs=None, stream=None):
    """Eq. 6 selection functions with the Delta branch left low-rank: u [B, K, D, H*W] ->
    (z [B, K, R, L] float32, Bs, Cs [B, K, N, L] in u's dtype); WB, WC [K, N, D], Wz [K, R, D]."""
    for t, n in [(u, "u"), (WB, "WB"), (WC, "WC"), (Wz, "Wz")]:
        _dev(t, n)
    B, K, D, L = u.shape
    N, R = WB.shape[1], Wz.shape[1]
    if L != H * W or tuple(WB.shape) != (K, N, D) or tuple(WC.shape) != (K, N, D) or tuple(Wz.shape) != (K, R, D):
        raise ValueError("u [B,K,D,H*W], WB/WC [K,N,D], Wz [K,R,D] expected")
    if any(w.dtype != torch.float32 for w in (WB, WC, Wz)):
        raise ValueError("weights must be float32")
    z = torch.empty((B, K, R, L), dtype=torch.float32, device=u.device) if z is None else z
    Bs = torch.empty((B, K, N, L), dtype=u.dtype, device=u.device) if Bs is None else Bs
    Cs = torch.empty((B, K, N, L), dtype=u.dtype, device=u.device) if Cs is None else Cs
    for t, n, shp, dt in [(z, "z", (B, K, R, L), torch.float32), (Bs, "Bs", (B, K, N, L), u.dtype),
                          (Cs, "Cs", (B, K, N, L), u.dtype)]:
        _dev(t, n)
        if tuple(t.shape) != shp or t.dtype != dt:
            raise ValueError(f"{n} must be {dt} {shp}")
    _check(lib.vmb_selection_lowrank_fwd(_ptr(u), _ptr(WB), _ptr(WC), _ptr(Wz), _ptr(Bs), _ptr(Cs), _ptr(z),
                                         B, K, D, N, R, H, W, _dtype_code(u.dtype), _stream(stream)),
           "vmb_selection_lowrank_fwd")
    return z, Bs, Cs


@_on_its_stream
def vmb_selective_scan_lowrank_fwd(u, z, Wup, A, Bs, Cs, Dskip, delta_bias, H: int, W: int, *, y=None,
                                   flags: int = VMB_FLAG_SOFTPLUS, workspace=None, stream=None) -> torch.Tensor:
    """Full-channel selective scan whose raw Deltas are Wup z, formed inside the scan:
    z [B, K, R, H*W] float32, Wup [K, D, R] float32; returns y [B, K, D, H*W] (dtype of u)."""
    for t, n in [(z, "z"), (Wup, "Wup")]:
        _dev(t, n)
    B, K, D, L = u.shape
    R = z.shape[2]
    if tuple(z.shape) != (B, K, R, L) or z.dtype != torch.float32:
        raise ValueError("z must be float32 [B, K, R, H*W]")
    if tuple(Wup.shape) != (K, D, R) or Wup.dtype != torch.float32:
        raise ValueError("Wup must be float32 [K, D, R]")
    B, K, D, N, L = _scan_shapes(u, u, A, Bs, Cs, Dskip, delta_bias, H, W)
    if y is None:
        y = torch.empty_like(u)
    _dev(y, "y")
    if y.shape != u.shape or y.dtype != u.dtype:
        raise ValueError("y must match u")
    ws_bytes = vmb_scan_workspace_bytes(VMB_PATH_FULL, B, K, D, N, H, W, u.dtype)
    if workspace is None:
        workspace = _default_ws.get(ws_bytes, u.device)
    _check(lib.vmb_selective_scan_lowrank_fwd(_ptr(u), _ptr(z), _ptr(Wup), _ptr(A), _ptr(Bs), _ptr(Cs), _ptr(Dskip),
                                              _ptr(delta_bias), _ptr(y), B, K, D, N, R, H, W, flags,
                                              _dtype_code(u.dtype), _ptr(workspace), workspace.numel(),
                                              _stream(stream)), "vmb_selective_scan_lowrank_fwd")
    return y


@_on_its_stream
def vmb_mean_scan_lowrank_fwd(u, z, Wup, A, Bs, Cs, Dskip, delta_bias, H: int, W: int, *, y=None, ybar=None,
                              want_ybar: bool = False, flags: int = VMB_FLAG_SOFTPLUS, workspace=None, stream=None):
    """Channel-mean scan whose raw Deltas are Wup z, formed inside the scan: z [B, K, R, H*W]
    float32, Wup [K, D, R] float32; returns (y [B, K, D, L], ybar [B, K, L] fp32 or None)."""
    for t, n in [(z, "z"), (Wup, "Wup")]:
        _dev(t, n)
    B, K, D, L = u.shape
    R = z.shape[2]
    if tuple(z.shape) != (B, K, R, L) or z.dtype != torch.float32:
        raise ValueError("z must be float32 [B, K, R, H*W]")
    if tuple(Wup.shape) != (K, D, R) or Wup.dtype != torch.float32:
        raise ValueError("Wup must be float32 [K, D, R]")
    B, K, D, N, L = _scan_shapes(u, u, A, Bs, Cs, Dskip, delta_bias, H, W)
    if y is None:
        y = torch.empty_like(u)
    _dev(y, "y")
    if y.shape != u.shape or y.dtype != u.dtype:
        raise ValueError("y must match u")
    if ybar is None and want_ybar:
        ybar = torch.empty((B, K, L), dtype=torch.float32, device=u.device)
    if ybar is not None:
        _dev(ybar, "ybar")
        if tuple(ybar.shape) != (B, K, L) or ybar.dtype != torch.float32:
            raise ValueError("ybar must be float32 [B, K, L]")
    ws_bytes = vmb_scan_workspace_bytes(VMB_PATH_MEAN, B, K, D, N, H, W, u.dtype)
    if workspace is None:
        workspace = _default_ws.get(ws_bytes, u.device)
    _check(lib.vmb_mean_scan_lowrank_fwd(_ptr(u), _ptr(z), _ptr(Wup), _ptr(A), _ptr(Bs), _ptr(Cs), _ptr(Dskip),
                                         _ptr(delta_bias), _ptr(y), _ptr(ybar),
                                         B, K, D, N, R, H, W, flags, _dtype_code(u.dtype), _ptr(workspace),
                                         workspace.numel(), _stream(stream)), "vmb_mean_scan_lowrank_fwd")
    return y, ybar


def vmb_mean_scan_bwd_workspace_bytes(B: int, K: int, D: int, N: int, H: int, W: int, groups: int = 1,
                                      dtype: torch.dtype = torch.float32) -> int:
    return int(lib.vmb_mean_scan_bwd_workspace_bytes(B, K, D, N, H, W, groups, _dtype_code(dtype)))


@_on_its_stream
def vmb_mean_scan_bwd(u, delta, A, Bs, Cs, Dskip, delta_bias, gy, H: int, W: int, *, groups: int = 1,
                      saved=None, flags: int = VMB_FLAG_SOFTPLUS, workspace=None, stream=None) -> dict:
    """Gradients of the (grouped) channel-mean scan given gy = dLoss/dy [B, K, D, H*W]: returns
    dict(u, delta, A, Bs, Cs, Dskip, delta_bias) with the inputs' shapes (delta: the raw Delta).
    saved: the group means vmb_mean_scan_train_fwd kept for these inputs, or None (recomputed)."""
    B, K, D, N, L = _scan_shapes(u, delta, A, Bs, Cs, Dskip, delta_bias, H, W)
    _dev(gy, "gy")
    if gy.shape != u.shape or gy.dtype != u.dtype:
        raise ValueError("gy must match u")
    if groups < 1 or D % groups:
        raise ValueError("groups must be >= 1 and divide D")
    if saved is not None:
        _dev(saved, "saved")
        if tuple(saved.shape) != (B, K, groups, N + 1, L) or saved.dtype != torch.float32:
            raise ValueError("saved must be float32 [B, K, groups, N + 1, L]")
    out = dict(u=torch.empty_like(u), delta=torch.empty_like(u), A=torch.empty_like(A), Bs=torch.empty_like(Bs),
               Cs=torch.empty_like(Cs), Dskip=torch.empty_like(Dskip), delta_bias=torch.empty_like(delta_bias))
    ws_bytes = vmb_mean_scan_bwd_workspace_bytes(B, K, D, N, H, W, groups, u.dtype)
    if workspace is None:
        workspace = torch.empty(max(ws_bytes, 256), dtype=torch.uint8, device=u.device)
    _check(lib.vmb_mean_scan_bwd(_ptr(u), _ptr(delta), _ptr(A), _ptr(Bs), _ptr(Cs), _ptr(Dskip), _ptr(delta_bias),
                                 _ptr(gy), _ptr(saved), _ptr(out["u"]), _ptr(out["delta"]), _ptr(out["A"]), _ptr(out["Bs"]),
                                 _ptr(out["Cs"]), _ptr(out["Dskip"]), _ptr(out["delta_bias"]), B, K, D, N, H, W,
                                 groups, flags, _dtype_code(u.dtype), _ptr(workspace), workspace.numel(),
                                 _stream(stream)), "vmb_mean_scan_bwd")
    return out


# ------------------------------------------- the channels-last token mixer

VMB_ACT_NONE, VMB_ACT_SILU, VMB_ACT_GELU = 0, 1, 2
VMB_ROTARY_INTERLEAVED, VMB_ROTARY_INVERSE = 0x1, 0x2

_ACTS = {"none": VMB_ACT_NONE, "silu": VMB_ACT_SILU, "gelu": VMB_ACT_GELU}
# workspaces of their own: the scans' must keep what the scans left in theirs
_delta_ws = Workspace()
_norm_ws = Workspace()
_layer_ws = Workspace(header=256)


# (a step of one token takes 2.5 us on the device: the marshalling below keeps to what it needs)
def _stream_of(t: torch.Tensor, stream) -> int:
    return _raw_stream(t.device.index) if stream is None else stream.cuda_stream


@functools.lru_cache(maxsize=4096)
def _delta_bytes(device, *sizes) -> int:
    return lib.vmb_delta_rule_workspace_bytes(*sizes)


@functools.lru_cache(maxsize=4096)
def _norm_bytes(device, *sizes) -> int:
    return lib.vmb_group_norm_workspace_bytes(*sizes)


@_on_its_stream
def delta_workspace(device=None, stream=None) -> torch.Tensor:
    """The default workspace of the calling thread's delta rule calls on a stream, the current one if none is given (for
    vmb_read_status; autograd runs backward passes in a thread of its own)."""
    return _delta_ws.get(256, torch.device("cuda" if device is None else device))


def _given(workspace, t):
    _dev(workspace, "workspace")
    _one_device(t, workspace)


def _heads(t: torch.Tensor, name: str):
    """(batch stride, token stride) of [B, T, H, D] whose heads and channels are dense."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    if t.dim() != 4:
        raise ValueError(f"{name} must be [B, T, heads, channels]")
    (B, T, H, D), (sb, st, sh, sd) = t.shape, t.stride()
    if (sd != 1 and D > 1) or (sh != D and H > 1):
        raise ValueError(f"{name}: the heads and channels of a token must be dense")
    return (sb if B > 1 else 0), (st if T > 1 else H * D)


def _delta_inputs(q, k, v, g, beta):
    """Checked sizes (B, T, Hk, Hv, Dk, Dv), dtype code and strides (None: dense) of the delta rule's inputs."""
    dt = q.dtype
    code = _dtype_code(dt)
    if k.dtype != dt or v.dtype != dt or g.dtype != dt or beta.dtype != dt:
        raise ValueError("q, k, v, g, beta must share one dtype")
    if not (q.is_cuda and k.is_cuda and v.is_cuda and g.is_cuda and beta.is_cuda):
        raise ValueError("q, k, v, g, beta must be CUDA tensors")
    if q.dim() != 4 or v.dim() != 4 or k.shape != q.shape:
        raise ValueError("q, k [B, T, Hk, Dk] and v [B, T, Hv, Dv] expected")
    if q.is_contiguous() and k.is_contiguous() and v.is_contiguous():
        strides = None
    else:
        strides = (ctypes.c_int64 * 6)(*_heads(q, "q"), *_heads(k, "k"), *_heads(v, "v"))
    B, T, Hk, Dk = q.shape
    vB, vT, Hv, Dv = v.shape
    if vB != B or vT != T:
        raise ValueError("q, k [B, T, Hk, Dk] and v [B, T, Hv, Dv] expected")
    if Hk < 1 or Hv % Hk:
        raise ValueError("the value heads must be a multiple of the key heads")
    if g.shape != (B, T, Hv) or beta.shape != g.shape:
        raise ValueError("g and beta must be [B, T, Hv]")
    if not (g.is_contiguous() and beta.is_contiguous()):
        raise ValueError("g and beta must be contiguous")
    return B, T, Hk, Hv, Dk, Dv, code, strides


def _delta_packed(offsets, max_len, B, T):
    """(sequences, longest, tokens) of dense [B, T] or packed [1, tokens] inputs."""
    if offsets is None:
        return B, T, B * T
    _dev(offsets, "offsets")
    if B != 1 or offsets.dim() != 1 or offsets.numel() < 1 or offsets.dtype != torch.int32:
        raise ValueError("packed sequences: a batch dimension of 1 and int32 offsets [sequences + 1] expected")
    if max_len is None or max_len < 0:
        raise ValueError("packed sequences: max_len, a bound of the longest sequence, is needed")
    return offsets.numel() - 1, min(int(max_len), T), T


def _scale(scale, Dk):
    return max(Dk, 1) ** -0.5 if scale is None else scale


def _state(t, name, shape):
    if t is not None:
        _dev(t, name)
        if t.shape != shape or t.dtype != torch.float32:
            raise ValueError(f"{name} must be float32 {tuple(shape)}")
    return t


def vmb_delta_rule_workspace_bytes(B: int, T: int, total: int, packed: bool, Hk: int, Hv: int, Dk: int, Dv: int,
                                   grads: bool = False, dtype: torch.dtype = torch.float32) -> int:
    return int(lib.vmb_delta_rule_workspace_bytes(B, T, total, int(packed), Hk, Hv, Dk, Dv, int(grads), _dtype_code(dtype)))


def vmb_delta_rule_saved_bytes(B: int, T: int, total: int, packed: bool, Hv: int, Dk: int, Dv: int,
                               dtype: torch.dtype = torch.float32) -> int:
    return int(lib.vmb_delta_rule_saved_bytes(B, T, total, int(packed), Hv, Dk, Dv, _dtype_code(dtype)))


@_on_its_stream
def vmb_delta_rule_fwd(q, k, v, g, beta, *, initial_state=None, offsets=None, max_len=None, scale=None,
                       want_state: bool = False, want_saved: bool = False, o=None, final_state=None, saved=None,
                       workspace=None, stream=None):
    """Gated delta rule over the tokens of every head: q, k [B, T, Hk, Dk], v [B, T, Hv, Dv] (rows of tokens may be
    strided), g (log decay), beta [B, T, Hv], initial_state [B, Hv, Dk, Dv] float32 or None; packed sequences with
    `offsets` int32 [sequences + 1] and `max_len` (the batch dimension is then 1, states are per sequence, and o is zero in
    rows that no sequence holds, as the gradients are).  `scale`
    defaults to Dk ** -0.5.  Returns (o [B, T, Hv, Dv], final_state or None, saved or None); `saved` is what
    vmb_delta_rule_bwd needs."""
    B, T, Hk, Hv, Dk, Dv, code, strides = _delta_inputs(q, k, v, g, beta)
    N, longest, total = _delta_packed(offsets, max_len, B, T)
    shape = (N, Hv, Dk, Dv)
    _state(initial_state, "initial_state", shape)
    if final_state is None and want_state:
        final_state = torch.empty(shape, dtype=torch.float32, device=q.device)
    _state(final_state, "final_state", shape)
    if o is None:
        o = torch.empty_like(v) if strides is None else v.new_empty((B, T, Hv, Dv))
    else:
        _dev(o, "o")
        if o.shape != (B, T, Hv, Dv) or o.dtype != q.dtype:
            raise ValueError("o must be [B, T, Hv, Dv] in the dtype of q")
    if not (N and Dk):
        o.zero_()  # (no sequences, or keys without channels: nothing is launched)
    if saved is None and want_saved:
        n = lib.vmb_delta_rule_saved_bytes(N, longest, total, offsets is not None, Hv, Dk, Dv, code)
        saved = torch.empty(n, dtype=torch.uint8, device=q.device)
    elif saved is not None:
        _saved_bytes(saved, N, longest, total, offsets, Hv, Dk, Dv, code)
    _one_device(q, k, v, g, beta, initial_state, offsets, o, final_state, saved)
    if workspace is None:
        dev = q.device
        workspace = _delta_ws.get(_delta_bytes(dev.index, N, longest, total, offsets is not None, Hk, Hv, Dk, Dv, 0, code), dev)
    else:
        _given(workspace, q)
    _check(lib.vmb_delta_rule_fwd(q.data_ptr(), k.data_ptr(), v.data_ptr(), g.data_ptr(), beta.data_ptr(), strides,
                                  _ptr(initial_state), _ptr(offsets), o.data_ptr(), _ptr(final_state), _ptr(saved), N,
                                  longest, total, Hk, Hv, Dk, Dv, _scale(scale, Dk), code,
                                  workspace.data_ptr(), workspace.numel(), _stream_of(q, stream)), "vmb_delta_rule_fwd")
    return o, final_state, saved


def _saved_bytes(saved, N, longest, total, offsets, Hv, Dk, Dv, code):
    _dev(saved, "saved")
    n = lib.vmb_delta_rule_saved_bytes(N, longest, total, offsets is not None, Hv, Dk, Dv, code)
    if saved.dtype != torch.uint8 or saved.numel() < n:
        raise ValueError(f"saved must be uint8 with at least {n} bytes")


@_on_its_stream
def vmb_delta_rule_bwd(q, k, v, g, beta, do, saved, *, dfinal_state=None, offsets=None, max_len=None, scale=None,
                       want_initial: bool = False, workspace=None, stream=None) -> dict:
    """Gradients of vmb_delta_rule_fwd given do = dLoss/do [B, T, Hv, Dv] and, optionally, dfinal_state: returns
    dict(q, k, v, g, beta[, initial_state]).  `saved`: the forward's, for the same inputs."""
    B, T, Hk, Hv, Dk, Dv, code, strides = _delta_inputs(q, k, v, g, beta)
    N, longest, total = _delta_packed(offsets, max_len, B, T)
    shape = (N, Hv, Dk, Dv)
    _state(dfinal_state, "dfinal_state", shape)
    _dev(do, "do")
    if do.shape != (B, T, Hv, Dv) or do.dtype != q.dtype:
        raise ValueError("do must be [B, T, Hv, Dv] in the dtype of q")
    _saved_bytes(saved, N, longest, total, offsets, Hv, Dk, Dv, code)
    dev = q.device
    new = torch.empty if N and Hv and Dk and Dv else torch.zeros  # (an empty problem launches nothing)
    out = {n: new(t.shape, dtype=q.dtype, device=dev) for n, t in (("q", q), ("k", k), ("v", v), ("g", g), ("beta", beta))}
    if want_initial:
        out["initial_state"] = torch.empty(shape, dtype=torch.float32, device=dev)
    _one_device(q, k, v, g, beta, do, saved, dfinal_state, offsets)
    if workspace is None:
        workspace = _delta_ws.get(_delta_bytes(dev.index, N, longest, total, offsets is not None, Hk, Hv, Dk, Dv, 1, code), dev)
    else:
        _given(workspace, q)
    _check(lib.vmb_delta_rule_bwd(q.data_ptr(), k.data_ptr(), g.data_ptr(), beta.data_ptr(), strides, _ptr(offsets),
                                  do.data_ptr(), _ptr(dfinal_state), saved.data_ptr(), out["q"].data_ptr(),
                                  out["k"].data_ptr(), out["v"].data_ptr(), out["g"].data_ptr(), out["beta"].data_ptr(),
                                  _ptr(out.get("initial_state")), N, longest, total, Hk, Hv, Dk, Dv,
                                  _scale(scale, Dk), code, workspace.data_ptr(), workspace.numel(),
                                  _stream_of(q, stream)), "vmb_delta_rule_bwd")
    return out


@_on_its_stream
def vmb_delta_rule_step(q, k, v, g, beta, state, *, slots=None, scale=None, o=None, stream=None) -> torch.Tensor:
    """The recurrence for T tokens (one, or a few) of every row from its state, updated in place: q, k [B, T, Hk, Dk],
    v [B, T, Hv, Dv], g, beta [B, T, Hv], state float32 [pool, Hv, Dk, Dv]; slots int32 [B] (row b uses state
    slots[b]; a negative slot is padding, its o is zero) or None (row b uses state b).  Returns o [B, T, Hv, Dv]."""
    B, T, Hk, Hv, Dk, Dv, code, strides = _delta_inputs(q, k, v, g, beta)
    _dev(state, "state")
    pool = state.shape[0]
    if state.shape != (pool, Hv, Dk, Dv) or state.dtype != torch.float32:
        raise ValueError("state must be float32 [pool, Hv, Dk, Dv]")
    if slots is not None:
        _dev(slots, "slots")
        if slots.shape != (B,) or slots.dtype != torch.int32:
            raise ValueError("slots must be int32 [B]")
    if o is None:
        o = torch.empty_like(v) if strides is None else v.new_empty((B, T, Hv, Dv))
    else:
        _dev(o, "o")
        if o.shape != (B, T, Hv, Dv) or o.dtype != q.dtype:
            raise ValueError("o must be [B, T, Hv, Dv] in the dtype of q")
    _one_device(q, k, v, g, beta, state, slots, o)
    if not Dk:
        o.zero_()
    _check(lib.vmb_delta_rule_step(q.data_ptr(), k.data_ptr(), v.data_ptr(), g.data_ptr(), beta.data_ptr(), strides,
                                   state.data_ptr(), _ptr(slots), o.data_ptr(), B, T, Hk, Hv, Dk, Dv, pool,
                                   _scale(scale, Dk), code, _stream_of(q, stream)), "vmb_delta_rule_step")
    return o


@functools.lru_cache(maxsize=256)
def _ints(values):
    return (ctypes.c_int * len(values))(*values)


def _rotary_out(x, out, name, dense):
    if out is None:
        return torch.empty_like(x) if dense else torch.empty(x.shape, dtype=x.dtype, device=x.device)
    _dev(out, name)
    if out.shape != x.shape or out.dtype != x.dtype:
        raise ValueError(f"{name} must have the shape and dtype of its input")
    return out


@_on_its_stream
def vmb_rotary_fwd(q, k, freq, positions=None, *, sections, grid=None, interleaved: bool = False,
                   inverse: bool = False, q_out=None, k_out=None, stream=None):
    """Rotary positions with len(sections) axes on q [B, T, Hq, D] and k [B, T, Hk, D] (or None; rows of tokens may be
    strided): sections gives each axis' pairs of channels, freq float32 [sum(sections)] the angle per position of
    every pair, positions int32 [axes, B, T] the tokens' places, or `grid` the sizes of the axes when the tokens lie
    in that row-major grid.  inverse: the opposite angles (the gradient).  Returns (q_out, k_out or None)."""
    code = _dtype_code(q.dtype)
    dense = q.is_contiguous() and (k is None or k.is_contiguous())
    if dense and q.dim() == 4:
        strides = None
        _dev(q, "q")
    else:
        strides = (ctypes.c_int64 * 4)(*_heads(q, "q"), *((0, 0) if k is None else _heads(k, "k")))
    B, T, Hq, D = q.shape
    Hk = 0
    if k is not None:
        if not k.is_cuda or k.dim() != 4 or k.dtype != q.dtype or k.shape[:2] != q.shape[:2] or k.shape[3] != D:
            raise ValueError("k must be [B, T, Hk, D] with the dtype, B, T and D of q")
        Hk = k.shape[2]
    _dev(freq, "freq")
    axes = len(sections)
    if not 1 <= axes <= 4:
        raise ValueError("one to four axes")
    if freq.dtype != torch.float32 or freq.dim() != 1 or freq.shape[0] != sum(sections):
        raise ValueError("freq must be float32 [sum(sections)]")
    if positions is not None:
        _dev(positions, "positions")
        if positions.dtype != torch.int32 or positions.shape != (axes, B, T):
            raise ValueError("positions must be int32 [axes, B, T]")
        cells = None
    else:
        if grid is None or len(grid) != axes:
            raise ValueError("positions, or a grid with one size for each axis, is needed")
        cells = _ints(tuple(grid))
    q_out = _rotary_out(q, q_out, "q_out", strides is None)
    if k is not None:
        k_out = _rotary_out(k, k_out, "k_out", strides is None)
    _one_device(q, k, freq, positions, q_out, k_out)
    flags = (VMB_ROTARY_INTERLEAVED if interleaved else 0) | (VMB_ROTARY_INVERSE if inverse else 0)
    _check(lib.vmb_rotary_fwd(q.data_ptr(), _ptr(k), freq.data_ptr(), _ptr(positions), q_out.data_ptr(), _ptr(k_out), B,
                              T, Hq, Hk, D, axes, _ints(tuple(sections)), cells, strides, flags, code,
                              _stream_of(q, stream)), "vmb_rotary_fwd")
    return q_out, k_out


def vmb_group_norm_workspace_bytes(B: int, L: int, C: int, groups: int, grads: bool = False,
                                   dtype: torch.dtype = torch.float32) -> int:
    return int(lib.vmb_group_norm_workspace_bytes(B, L, C, groups, int(grads), _dtype_code(dtype)))


def _norm_inputs(x, weight, bias, groups, act):
    _dev(x, "x")
    if x.dim() < 2:
        raise ValueError("x must be [B, ..., C]")
    B, C = x.shape[0], x.shape[-1]
    if groups < 1 or C % groups:
        raise ValueError("groups must be >= 1 and divide the channels")
    for t, n in ((weight, "weight"), (bias, "bias")):
        if t is not None:
            _dev(t, n)
            if t.shape != (C,) or t.dtype != torch.float32:
                raise ValueError(f"{n} must be float32 [C]")
    if act not in _ACTS:
        raise ValueError(f"act must be one of {sorted(_ACTS)}")
    L = x.numel() // (B * C) if B * C else 0
    return B, L, C, _dtype_code(x.dtype), _ACTS[act]


@_on_its_stream
def vmb_group_norm_fwd(x, weight, bias, groups: int, *, eps: float = 1e-5, act: str = "none", want_stats: bool = False,
                       y=None, stats=None, workspace=None, stream=None):
    """Group norm with an activation ("none", "silu", "gelu"), channels last: x [B, ..., C], weight and bias float32
    [C] or None.  Returns (y, stats [B, groups, 2] float32 (mean, 1 / sqrt(variance + eps)) or None)."""
    B, L, C, code, a = _norm_inputs(x, weight, bias, groups, act)
    if y is None:
        y = torch.empty_like(x)
    else:
        _dev(y, "y")
        if y.shape != x.shape or y.dtype != x.dtype:
            raise ValueError("y must match x")
    if stats is None and want_stats:
        stats = torch.empty((B, groups, 2), dtype=torch.float32, device=x.device)
    _state(stats, "stats", (B, groups, 2))
    if workspace is None:
        workspace = _norm_ws.get(_norm_bytes(x.device.index, B, L, C, groups, 0, code), x.device)
    else:
        _given(workspace, x)
    _one_device(x, weight, bias, y, stats)
    _check(lib.vmb_group_norm_fwd(x.data_ptr(), _ptr(weight), _ptr(bias), y.data_ptr(), _ptr(stats), B, L, C, groups, eps,
                                  a, code, workspace.data_ptr(), workspace.numel(), _stream_of(x, stream)), "vmb_group_norm_fwd")
    return y, stats


@_on_its_stream
def vmb_group_norm_bwd(x, weight, bias, stats, dy, groups: int, *, act: str = "none", workspace=None, stream=None) -> dict:
    """Gradients of vmb_group_norm_fwd given dy and the forward's stats: dict(x, weight, bias), the latter two float32
    [C] (None where the input was None)."""
    B, L, C, code, a = _norm_inputs(x, weight, bias, groups, act)
    _dev(dy, "dy")
    if dy.shape != x.shape or dy.dtype != x.dtype:
        raise ValueError("dy must match x")
    if stats is None:
        raise ValueError("the forward's stats are needed")
    _state(stats, "stats", (B, groups, 2))
    new = torch.empty_like if x.numel() else torch.zeros_like  # (an empty problem launches nothing: sums of nothing)
    out = dict(x=torch.empty_like(x), weight=None if weight is None else new(weight), bias=None if bias is None else new(bias))
    if workspace is None:
        workspace = _norm_ws.get(_norm_bytes(x.device.index, B, L, C, groups, 1, code), x.device)
    else:
        _given(workspace, x)
    _one_device(x, weight, bias, stats, dy)
    _check(lib.vmb_group_norm_bwd(x.data_ptr(), _ptr(weight), _ptr(bias), stats.data_ptr(), dy.data_ptr(),
                                  out["x"].data_ptr(), _ptr(out["weight"]), _ptr(out["bias"]), B, L, C, groups, a, code,
                                  workspace.data_ptr(), workspace.numel(), _stream_of(x, stream)), "vmb_group_norm_bwd")
    return out


# ---------------------------------------------------------------- a layer around a scan over tokens


def _rows(t, name: str, B: int, T: int, C: int, dtype):
    """(batch stride, token stride) of [B, T, C] of the given type whose channels are dense."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    if t.shape != (B, T, C) or t.dtype != dtype:
        raise ValueError(f"{name} must be [{B}, {T}, {C}] in the dtype of x")
    sb, st, sc = t.stride()
    if sc != 1 and C > 1:
        raise ValueError(f"{name}: the channels of a token must be dense")
    return (sb if B > 1 else 0), (st if T > 1 else C)


def _float(t, name: str, shape):
    if t is not None:
        _dev(t, name)
        if t.shape != shape or t.dtype != torch.float32:
            raise ValueError(f"{name} must be float32 {list(shape)}")


def _like(t, name: str, shape, dtype):
    """A given dense tensor (or None) of this shape and type."""
    if t is not None:
        _dev(t, name)
        if t.shape != shape or t.dtype != dtype:
            raise ValueError(f"{name} must be {list(shape)} in the dtype of x")


def _empty(x, dense):
    """A dense tensor like x (one call into torch where x is dense itself)."""
    return torch.empty_like(x) if dense else torch.empty(x.shape, dtype=x.dtype, device=x.device)


def _sequences(offsets, B, T):
    """(sequences, their length, tokens) of dense [B, T] or packed [1, tokens] inputs."""
    if offsets is None:
        return B, T, B * T
    _dev(offsets, "offsets")
    if B != 1 or offsets.dim() != 1 or offsets.numel() < 1 or offsets.dtype != torch.int32:
        raise ValueError("packed sequences: a batch dimension of 1 and int32 offsets [sequences + 1] expected")
    return offsets.numel() - 1, T, T


def _pool(state, slots, B):
    if slots is None:
        if state.shape[0] < B:
            raise ValueError("state: fewer rows than the batch, and no slots")
        return
    _dev(slots, "slots")
    if slots.shape != (B,) or slots.dtype != torch.int32:
        raise ValueError("slots must be int32 [B]")


@functools.lru_cache(maxsize=4096)
def _layer_bytes(device, name, *sizes) -> int:
    return getattr(lib, name)(*sizes)


def _layer_workspace(workspace, t, name, *sizes):
    if workspace is None:
        return _layer_ws.get(_layer_bytes(t.device.index, name, *sizes), t.device)
    _given(workspace, t)
    return workspace


@_on_its_stream
def layer_workspace(device=None, stream=None) -> torch.Tensor:
    """The default workspace of the calling thread's convolutions, scans over tokens, norms and products on a stream, the
    current one if none is given (for vmb_read_status)."""
    return _layer_ws.get(256, torch.device("cuda" if device is None else device))


def vmb_causal_conv_workspace_bytes(B: int, T: int, total: int, packed: bool, C: int, W: int,
                                    dtype: torch.dtype = torch.float32) -> int:
    return int(lib.vmb_causal_conv_workspace_bytes(B, T, total, int(packed), C, W, _dtype_code(dtype)))


def _conv_inputs(x, weight, bias, act):
    code = _dtype_code(x.dtype)
    if x.dim() != 3 or weight.dim() != 2:
        raise ValueError("x [B, T, C] and weight [C, W] expected")
    B, T, C = x.shape
    W = weight.shape[1]
    strides = _rows(x, "x", B, T, C, x.dtype)
    _float(weight, "weight", (C, W))
    _float(bias, "bias", (C,))
    if act not in ("none", "silu"):
        raise ValueError("act must be 'none' or 'silu'")
    return B, T, C, W, code, _ACTS[act], (None if x.is_contiguous() else (ctypes.c_int64 * 2)(*strides))


@_on_its_stream
def vmb_causal_conv_fwd(x, weight, bias=None, *, act: str = "silu", initial_state=None, offsets=None, want_state: bool = False,
                        y=None, final_state=None, stream=None):
    """Short causal convolution along the tokens, one filter per channel, with an activation ("silu" or "none"): x
    [B, T, C] (rows of tokens may be strided), weight float32 [C, W], bias float32 [C] or None, initial_state
    [B, W - 1, C] or None (zeros); packed sequences with `offsets` int32 [sequences + 1] (the batch dimension is then 1,
    states are per sequence, rows that no sequence holds are zero).  Returns (y [B, T, C], final_state or None)."""
    B, T, C, W, code, a, strides = _conv_inputs(x, weight, bias, act)
    n, T1, total = _sequences(offsets, B, T)
    _like(initial_state, "initial_state", (n, W - 1, C), x.dtype)
    if final_state is None and want_state:
        final_state = x.new_empty((n, W - 1, C))
    _like(final_state, "final_state", (n, W - 1, C), x.dtype)
    if y is None:
        y = _empty(x, strides is None)
    else:
        _like(y, "y", (B, T, C), x.dtype)
    _one_device(x, weight, bias, initial_state, offsets, y, final_state)
    _check(lib.vmb_causal_conv_fwd(x.data_ptr(), weight.data_ptr(), _ptr(bias), strides, _ptr(initial_state), _ptr(offsets),
                                   y.data_ptr(), _ptr(final_state), n, T1, total, C, W, a, code, _stream_of(x, stream)),
           "vmb_causal_conv_fwd")
    return y, final_state


@_on_its_stream
def vmb_causal_conv_bwd(x, weight, bias, dy, *, act: str = "silu", initial_state=None, dfinal_state=None, offsets=None,
                        want_initial: bool = False, workspace=None, stream=None) -> dict:
    """Gradients of vmb_causal_conv_fwd given dy [B, T, C] and, optionally, dfinal_state: dict(x, weight, bias (None without
    one)[, initial_state])."""
    B, T, C, W, code, a, strides = _conv_inputs(x, weight, bias, act)
    n, T1, total = _sequences(offsets, B, T)
    _like(initial_state, "initial_state", (n, W - 1, C), x.dtype)
    _like(dfinal_state, "dfinal_state", (n, W - 1, C), x.dtype)
    if dy is None:
        raise ValueError("dy is needed")
    _like(dy, "dy", (B, T, C), x.dtype)
    out = dict(x=x.new_empty((B, T, C)), weight=torch.empty_like(weight), bias=None if bias is None else torch.empty_like(bias))
    if want_initial:
        out["initial_state"] = x.new_empty((n, W - 1, C))
    _one_device(x, weight, bias, dy, initial_state, dfinal_state, offsets)
    ws = _layer_workspace(workspace, x, "vmb_causal_conv_workspace_bytes", n, T1, total, offsets is not None, C, W, code)
    _check(lib.vmb_causal_conv_bwd(x.data_ptr(), weight.data_ptr(), _ptr(bias), strides, _ptr(initial_state), _ptr(offsets),
                                   dy.data_ptr(), _ptr(dfinal_state), out["x"].data_ptr(), out["weight"].data_ptr(),
                                   _ptr(out["bias"]), _ptr(out.get("initial_state")), n, T1, total, C, W, a, code,
                                   ws.data_ptr(), ws.numel(), _stream_of(x, stream)), "vmb_causal_conv_bwd")
    return out


@_on_its_stream
def vmb_causal_conv_step(x, weight, bias, state, *, act: str = "silu", slots=None, y=None, stream=None) -> torch.Tensor:
    """T tokens (one, or a few) of every row from the inputs kept in its state, which move on in place: x [B, T, C], state
    [pool, W - 1, C]; slots int32 [B] (row b uses state slots[b]; a negative slot is padding, its y is zero) or None (row
    b uses state b).  Returns y [B, T, C]."""
    B, T, C, W, code, a, strides = _conv_inputs(x, weight, bias, act)
    if state.dim() != 3:
        raise ValueError("state must be [pool, W - 1, C]")
    _like(state, "state", (state.shape[0], W - 1, C), x.dtype)
    _pool(state, slots, B)
    if y is None:
        y = _empty(x, strides is None)
    else:
        _like(y, "y", (B, T, C), x.dtype)
    _one_device(x, weight, bias, state, slots, y)
    _check(lib.vmb_causal_conv_step(x.data_ptr(), weight.data_ptr(), _ptr(bias), strides, state.data_ptr(), _ptr(slots),
                                    y.data_ptr(), B, T, C, W, state.shape[0], a, code, _stream_of(x, stream)),
           "vmb_causal_conv_step")
    return y


def vmb_token_scan_workspace_bytes(B: int, T: int, total: int, packed: bool, D: int, N: int, grads: bool = False,
                                   dtype: torch.dtype = torch.float32) -> int:
    return int(lib.vmb_token_scan_workspace_bytes(B, T, total, int(packed), D, N, int(grads), _dtype_code(dtype)))


def vmb_token_scan_saved_bytes(B: int, T: int, total: int, packed: bool, D: int, N: int) -> int:
    return int(lib.vmb_token_scan_saved_bytes(B, T, total, int(packed), D, N))


def _token_scan_inputs(x, delta, A, Bm, Cm, Dskip, delta_bias, z):
    dtype = x.dtype
    code = _dtype_code(dtype)
    if x.dim() != 3 or A.dim() != 2:
        raise ValueError("x [B, T, D] and A [D, N] expected")
    B, T, D = shape = x.shape
    N = A.shape[1]
    _float(A, "A", (D, N))
    _float(Dskip, "Dskip", (D,))
    _float(delta_bias, "delta_bias", (D,))
    states = (B, T, N)
    if (x.is_contiguous() and delta.is_contiguous() and Bm.is_contiguous() and Cm.is_contiguous() and (z is None or z.is_contiguous())
            and x.is_cuda and delta.is_cuda and Bm.is_cuda and Cm.is_cuda and (z is None or z.is_cuda)
            and delta.shape == shape and Bm.shape == states and Cm.shape == states and (z is None or z.shape == shape)
            and delta.dtype == dtype and Bm.dtype == dtype and Cm.dtype == dtype and (z is None or z.dtype == dtype)):
        return B, T, D, N, code, None
    strides = [*_rows(x, "x", B, T, D, dtype), *_rows(delta, "delta", B, T, D, dtype),
               *_rows(Bm, "Bm", B, T, N, dtype), *_rows(Cm, "Cm", B, T, N, dtype)]
    strides += [0, 0] if z is None else _rows(z, "z", B, T, D, dtype)
    return B, T, D, N, code, (ctypes.c_int64 * 10)(*strides)


def _token_scan_saved(saved, n, T, total, packed, D, N):
    need = lib.vmb_token_scan_saved_bytes(n, T, total, packed, D, N)
    if saved is True:
        return need
    _dev(saved, "saved")
    if saved.dtype != torch.uint8 or saved.numel() < need:
        raise ValueError(f"saved must be uint8 with at least {need} bytes")


@_on_its_stream
def vmb_token_scan_fwd(x, delta, A, Bm, Cm, Dskip=None, delta_bias=None, z=None, *, softplus: bool = True, initial_state=None,
                       offsets=None, want_state: bool = False, want_saved: bool = False, y=None, final_state=None, saved=None,
                       workspace=None, stream=None):
    """Selective scan over tokens with its gate: x, delta, z (or None) [B, T, D], Bm, Cm [B, T, N] (rows of tokens may be
    strided), A float32 [D, N], Dskip, delta_bias float32 [D] or None, initial_state float32 [B, D, N] or None (zeros);
    packed sequences with `offsets` int32 [sequences + 1] (the batch dimension is then 1, states are per sequence, rows that
    no sequence holds are zero).  Returns (y [B, T, D], final_state or None, saved or None); `saved` is what
    vmb_token_scan_bwd needs."""
    B, T, D, N, code, strides = _token_scan_inputs(x, delta, A, Bm, Cm, Dskip, delta_bias, z)
    n, T1, total = _sequences(offsets, B, T)
    packed = offsets is not None
    _float(initial_state, "initial_state", (n, D, N))
    if final_state is None and want_state:
        final_state = torch.empty((n, D, N), dtype=torch.float32, device=x.device)
    _float(final_state, "final_state", (n, D, N))
    if y is None:
        y = _empty(x, x.is_contiguous())
    else:
        _like(y, "y", (B, T, D), x.dtype)
    if saved is not None:
        _token_scan_saved(saved, n, T1, total, packed, D, N)
    elif want_saved:
        saved = torch.empty(_token_scan_saved(True, n, T1, total, packed, D, N), dtype=torch.uint8, device=x.device)
    _one_device(x, delta, A, Bm, Cm, Dskip, delta_bias, z, initial_state, offsets, y, final_state, saved)
    ws = _layer_workspace(workspace, x, "vmb_token_scan_workspace_bytes", n, T1, total, packed, D, N, 0, code)
    _check(lib.vmb_token_scan_fwd(x.data_ptr(), delta.data_ptr(), A.data_ptr(), Bm.data_ptr(), Cm.data_ptr(), _ptr(Dskip),
                                  _ptr(delta_bias), _ptr(z), strides, _ptr(initial_state), _ptr(offsets), y.data_ptr(),
                                  _ptr(final_state), _ptr(saved), n, T1, total, D, N, VMB_FLAG_SOFTPLUS if softplus else 0, code,
                                  ws.data_ptr(), ws.numel(), _stream_of(x, stream)), "vmb_token_scan_fwd")
    return y, final_state, saved


@_on_its_stream
def vmb_token_scan_bwd(x, delta, A, Bm, Cm, Dskip, delta_bias, z, dy, saved, *, softplus: bool = True, dfinal_state=None,
                       offsets=None, want_initial: bool = False, workspace=None, stream=None) -> dict:
    """Gradients of vmb_token_scan_fwd given dy [B, T, D] and, optionally, dfinal_state: dict(x, delta, A, B, C, Dskip,
    delta_bias, z[, initial_state]), None where the input was None.  `saved`: the forward's, for the same inputs."""
    B, T, D, N, code, strides = _token_scan_inputs(x, delta, A, Bm, Cm, Dskip, delta_bias, z)
    n, T1, total = _sequences(offsets, B, T)
    packed = offsets is not None
    _float(dfinal_state, "dfinal_state", (n, D, N))
    if dy is None or saved is None:
        raise ValueError("dy and the forward's saved are needed")
    _like(dy, "dy", (B, T, D), x.dtype)
    _token_scan_saved(saved, n, T1, total, packed, D, N)
    dev = x.device
    out = {k: None if t is None else torch.empty(t.shape, dtype=t.dtype, device=dev)
           for k, t in (("x", x), ("delta", delta), ("A", A), ("B", Bm), ("C", Cm), ("Dskip", Dskip), ("delta_bias", delta_bias),
                        ("z", z))}
    if want_initial:
        out["initial_state"] = torch.empty((n, D, N), dtype=torch.float32, device=dev)
    _one_device(x, delta, A, Bm, Cm, Dskip, delta_bias, z, dy, saved, dfinal_state, offsets)
    ws = _layer_workspace(workspace, x, "vmb_token_scan_workspace_bytes", n, T1, total, packed, D, N, 1, code)
    _check(lib.vmb_token_scan_bwd(x.data_ptr(), delta.data_ptr(), A.data_ptr(), Bm.data_ptr(), Cm.data_ptr(), _ptr(Dskip),
                                  _ptr(delta_bias), _ptr(z), strides, _ptr(offsets), dy.data_ptr(), _ptr(dfinal_state),
                                  saved.data_ptr(), out["x"].data_ptr(), out["delta"].data_ptr(), out["A"].data_ptr(),
                                  out["B"].data_ptr(), out["C"].data_ptr(), _ptr(out["Dskip"]), _ptr(out["delta_bias"]),
                                  _ptr(out["z"]), _ptr(out.get("initial_state")), n, T1, total, D, N,
                                  VMB_FLAG_SOFTPLUS if softplus else 0, code, ws.data_ptr(), ws.numel(),
                                  _stream_of(x, stream)), "vmb_token_scan_bwd")
    return out


@_on_its_stream
def vmb_token_scan_step(x, delta, A, Bm, Cm, Dskip, delta_bias, z, state, *, softplus: bool = True, slots=None, y=None,
                        stream=None) -> torch.Tensor:
    """The scan for T tokens (one, or a few) of every row from its state, updated in place: inputs as for
    vmb_token_scan_fwd, state float32 [pool, D, N]; slots int32 [B] (row b uses state slots[b]; a negative slot is padding,
    its y is zero) or None (row b uses state b).  Returns y [B, T, D]."""
    B, T, D, N, code, strides = _token_scan_inputs(x, delta, A, Bm, Cm, Dskip, delta_bias, z)
    if state.dim() != 3:
        raise ValueError("state must be float32 [pool, D, N]")
    _float(state, "state", (state.shape[0], D, N))
    _pool(state, slots, B)
    if y is None:
        y = _empty(x, x.is_contiguous())
    else:
        _like(y, "y", (B, T, D), x.dtype)
    _one_device(x, delta, A, Bm, Cm, Dskip, delta_bias, z, state, slots, y)
    _check(lib.vmb_token_scan_step(x.data_ptr(), delta.data_ptr(), A.data_ptr(), Bm.data_ptr(), Cm.data_ptr(), _ptr(Dskip),
                                   _ptr(delta_bias), _ptr(z), strides, state.data_ptr(), _ptr(slots), y.data_ptr(), B, T, D, N,
                                   state.shape[0], VMB_FLAG_SOFTPLUS if softplus else 0, code, _stream_of(x, stream)),
           "vmb_token_scan_step")
    return y


def vmb_rms_norm_workspace_bytes(rows: int, C: int, dtype: torch.dtype = torch.float32) -> int:
    return int(lib.vmb_rms_norm_workspace_bytes(rows, C, _dtype_code(dtype)))


def _rms_inputs(x, weight):
    _dev(x, "x")
    if x.dim() < 1:
        raise ValueError("x must be [..., C]")
    C = x.shape[-1]
    _float(weight, "weight", (C,))
    return x.numel() // C if C else x.shape[:-1].numel(), C, _dtype_code(x.dtype)


@_on_its_stream
def vmb_rms_norm_fwd(x, weight=None, residual=None, *, eps: float = 1e-6, bits8: bool = False, want_stats: bool = False,
                     y=None, total=None, scale=None, rstd=None, stream=None):
    """Root-mean-square norm of the rows of x [..., C] after the residual's addition: returns (y, total, scale, rstd).
    total = x + residual in the dtype of x (None without a residual), y = total * rstd * weight (float32 [C] or None) in
    the dtype of x, or with `bits8` in torch.float8_e4m3fn, to be multiplied by scale (float32 [...], one per row; otherwise
    None); rstd float32 [...] with `want_stats`, for vmb_rms_norm_bwd."""
    rows, C, code = _rms_inputs(x, weight)
    lead, kind = x.shape[:-1], torch.float8_e4m3fn if bits8 else x.dtype
    _like(residual, "residual", x.shape, x.dtype)
    if y is None:
        y = torch.empty(x.shape, dtype=kind, device=x.device)
    else:
        _dev(y, "y")
        if y.shape != x.shape or y.dtype != kind:
            raise ValueError(f"y must be {list(x.shape)} in {kind}")
    if residual is None:
        if total is not None:
            raise ValueError("total: without a residual it is x")
    elif total is None:
        total = torch.empty_like(x)
    _like(total, "total", x.shape, x.dtype)
    if not bits8 and scale is not None:
        raise ValueError("scale: only 8-bit outputs have one")
    if bits8 and scale is None:
        scale = torch.empty(lead, dtype=torch.float32, device=x.device)
    if rstd is None and want_stats:
        rstd = torch.empty(lead, dtype=torch.float32, device=x.device)
    _float(scale, "scale", lead)
    _float(rstd, "rstd", lead)
    _one_device(x, weight, residual, y, total, scale, rstd)
    _check(lib.vmb_rms_norm_fwd(x.data_ptr(), _ptr(residual), _ptr(weight), y.data_ptr(), _ptr(total), _ptr(scale), _ptr(rstd),
                                rows, C, eps, code, _stream_of(x, stream)), "vmb_rms_norm_fwd")
    return y, total, scale, rstd


@_on_its_stream
def vmb_rms_norm_bwd(x, weight, rstd, dy, *, dsum=None, workspace=None, stream=None) -> dict:
    """Gradients of vmb_rms_norm_fwd given dy and, optionally, dsum, the gradient that reaches the sum on its own:
    dict(x, weight (None without one)).  x: what was normalised (the forward's total, if there was a residual); the
    gradient of the residual is that of x."""
    rows, C, code = _rms_inputs(x, weight)
    if rstd is None or dy is None:
        raise ValueError("dy and the forward's rstd are needed")
    _float(rstd, "rstd", x.shape[:-1])
    _like(dy, "dy", x.shape, x.dtype)
    _like(dsum, "dsum", x.shape, x.dtype)
    out = dict(x=torch.empty_like(x), weight=None if weight is None else torch.empty_like(weight))
    _one_device(x, weight, rstd, dy, dsum)
    ws = _layer_workspace(workspace, x, "vmb_rms_norm_workspace_bytes", rows, C, code)
    _check(lib.vmb_rms_norm_bwd(x.data_ptr(), _ptr(weight), rstd.data_ptr(), dy.data_ptr(), _ptr(dsum), out["x"].data_ptr(),
                                _ptr(out["weight"]), rows, C, code, ws.data_ptr(), ws.numel(), _stream_of(x, stream)),
           "vmb_rms_norm_bwd")
    return out


def vmb_linear_workspace_bytes(M: int, K: int, N: int, grads: bool = False) -> int:
    return int(lib.vmb_linear_workspace_bytes(M, K, N, int(grads)))


def _linear_inputs(x, weight, kind, act):
    """(rows, K, N, elements between rows) of x [..., K], whose rows may be strided evenly, and weight [N, K]."""
    if not x.is_cuda:
        raise ValueError("x must be a CUDA tensor")
    _dev(weight, "weight")
    if x.dim() < 1 or weight.dim() != 2 or x.shape[-1] != weight.shape[1]:
        raise ValueError("x [..., K] and weight [N, K] expected")
    if x.dtype != kind or weight.dtype != kind:
        raise TypeError(f"x and weight must be {kind}")
    if act not in _ACTS:
        raise ValueError(f"act must be one of {sorted(_ACTS)}")
    N, K = weight.shape
    if x.is_contiguous():
        return (x.numel() // K if K else x.shape[:-1].numel()), K, N, K
    try:
        flat = x.view(-1, K)
    except RuntimeError:
        raise ValueError("x: the rows must be evenly strided") from None
    if flat.stride(1) != 1 and K > 1:
        raise ValueError("x: the channels of a row must be dense")
    return flat.shape[0], K, N, (flat.stride(0) if flat.shape[0] > 1 else K)


@_on_its_stream
def vmb_linear_fwd(x, weight, bias=None, *, act: str = "none", residual=None, x_scale=None, weight_scale=None,
                   want_pre: bool = False, y=None, pre=None, workspace=None, stream=None):
    """Matrix product of a projection: y = act(x weight^T + bias) + residual in bfloat16, act "none", "silu" or "gelu".
    x [..., K] (rows may be strided evenly) and weight [N, K] bfloat16, or torch.float8_e4m3fn with x_scale float32 [...] and
    weight_scale float32 [N], the scales of their rows; bias float32 [N] or None; residual [..., N] bfloat16 or None.
    Returns (y [..., N], pre or None); pre = x weight^T + bias in bfloat16 with `want_pre`, for vmb_linear_bwd."""
    if (x_scale is None) != (weight_scale is None):
        raise ValueError("x_scale and weight_scale are given together")
    M, K, N, x_t = _linear_inputs(x, weight, torch.bfloat16 if x_scale is None else torch.float8_e4m3fn, act)
    lead = x.shape[:-1]
    shape = (*lead, N)
    _float(x_scale, "x_scale", lead)
    _float(weight_scale, "weight_scale", (N,))
    _float(bias, "bias", (N,))
    for t, name in ((residual, "residual"), (y, "y"), (pre, "pre")):
        if t is not None:
            _dev(t, name)
            if t.shape != shape or t.dtype != torch.bfloat16:
                raise ValueError(f"{name} must be bfloat16 {list(shape)}")
    if y is None:
        y = torch.empty(shape, dtype=torch.bfloat16, device=x.device)
    if pre is None and want_pre:
        pre = torch.empty(shape, dtype=torch.bfloat16, device=x.device)
    _one_device(x, weight, bias, residual, x_scale, weight_scale, y, pre)
    ws = _layer_workspace(workspace, x, "vmb_linear_workspace_bytes", M, K, N, 0)
    _check(lib.vmb_linear_fwd(x.data_ptr(), x_t, weight.data_ptr(), _ptr(x_scale), _ptr(weight_scale), _ptr(bias), _ptr(residual),
                              y.data_ptr(), _ptr(pre), M, K, N, _ACTS[act], ws.data_ptr(), ws.numel(), _stream_of(x, stream)),
           "vmb_linear_fwd")
    return y, pre


@_on_its_stream
def vmb_linear_bwd(x, weight, dy, pre=None, *, act: str = "none", want_x: bool = True, want_weight: bool = True,
                   want_bias: bool = False, workspace=None, stream=None) -> dict:
    """Gradients of vmb_linear_fwd of bfloat16 given dy [..., N] and, with an activation, the forward's pre: dict(x [..., K],
    weight [N, K] (bfloat16), bias (float32 [N])), None where not wanted; the residual's gradient is dy."""
    M, K, N, x_t = _linear_inputs(x, weight, torch.bfloat16, act)
    shape = (*x.shape[:-1], N)
    if dy is None or (pre is None and act != "none"):
        raise ValueError("dy and, with an activation, the forward's pre are needed")
    for t, name in ((dy, "dy"), (pre, "pre")):
        if t is not None:
            _dev(t, name)
            if t.shape != shape or t.dtype != torch.bfloat16:
                raise ValueError(f"{name} must be bfloat16 {list(shape)}")
    dev = x.device
    out = dict(x=torch.empty(x.shape, dtype=x.dtype, device=dev) if want_x else None,
               weight=torch.empty((N, K), dtype=x.dtype, device=dev) if want_weight else None,
               bias=torch.empty((N,), dtype=torch.float32, device=dev) if want_bias else None)
    _one_device(x, weight, dy, pre)
    ws = _layer_workspace(workspace, x, "vmb_linear_workspace_bytes", M, K, N, 1)
    _check(lib.vmb_linear_bwd(x.data_ptr(), x_t, weight.data_ptr(), _ptr(pre), dy.data_ptr(), _ptr(out["x"]), _ptr(out["weight"]),
                              _ptr(out["bias"]), M, K, N, _ACTS[act], ws.data_ptr(), ws.numel(), _stream_of(x, stream)),
           "vmb_linear_bwd")
    return out


@_on_its_stream
def vmb_read_status(workspace=None, device=None, stream=None) -> int:
    """Synchronise and return (then clear) the device error word of a workspace; without one, of all default workspaces that
    the calling thread's calls have used on the device: the scans', the delta rule's, and those of the layer around the scan
    over tokens (VMB_OK, or an error of one of them).  A call captured into a graph has a default workspace that nobody else
    can reach: give it one (`workspace=`) to read its status after a replay."""
    if workspace is not None:
        return int(lib.vmb_read_status(_ptr(workspace), _stream(stream)))
    dev = torch.device("cuda" if device is None else device)
    index = torch.cuda.current_device() if dev.index is None else dev.index
    _default_ws.get(256, dev)
    torch.cuda.synchronize(index)
    found = [int(lib.vmb_read_status(_ptr(buf), _stream(stream)))
             for kept in (_default_ws, _delta_ws, _layer_ws) for bufs in (kept.buffers(), kept.outgrown())
             for (i, _), buf in bufs.items() if i == index]
    return next((status for status in found if status != VMB_OK), VMB_OK)


@_on_its_stream
def default_workspace(device=None, stream=None) -> torch.Tensor:
    """The default workspace of the calling thread's scans on a stream (the current one if none is given)."""
    return _default_ws.get(256, torch.device("cuda" if device is None else device))
