"""ctypes binding of libtfno.so: argument marshalling only.

Every step of the spectral convolution runs inside the HIP library; PyTorch is used for device
allocation and streams.  The functions mirror the C ABI in ``include/tfno.h`` name for name.  There is
no CPU fallback: if the library has not been built, loading raises.
"""
from __future__ import annotations

import ctypes
import functools
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libtfno.so")

OK, ERR_NULL, ERR_SHAPE, ERR_UNSUPPORTED, ERR_ALIAS, ERR_WORKSPACE, ERR_HIP, ERR_ALIGN = range(8)

EXPORTS = (
    "tfno_spectral_conv1d",
    "tfno_spectral_conv2d",
    "tfno_spectral_conv1d_staged",
    "tfno_spectral_conv2d_staged",
    "tfno_spectral_conv1d_pruned",
    "tfno_spectral_conv1d_fft_gemm",
    "tfno_spectral_conv1d_gemm_ifft",
    "tfno_spectral_conv1d_auto",
    "tfno_spectral_conv2d_rect",
    "tfno_spectral_conv2d_rect_staged",
    "tfno_spectral_conv2d_permode",
    "tfno_spectral_conv1d_permode",
    "tfno_spectral_conv1d_real",
    "tfno_fno2d_real",
    "tfno_fno2d_real_workspace_bytes",
    "tfno_fno1d_real",
    "tfno_fno1d_real_workspace_bytes",
    "tfno_spectral_conv2d_noalloc",
    "tfno_spectral_conv2d_strips",
    "tfno_workspace_bytes",
    "tfno_workspace_bytes_2d",
    "tfno_set_workspace",
    "tfno_status_string",
    "tfno_version",
    "tfno_head_norm_rope",
    "tfno_head_norm_rope_backward",
    "tfno_head_norm_rope_workspace_bytes",
    "tfno_gated_delta_rule",
    "tfno_gated_delta_rule_backward",
    "tfno_gated_delta_rule_tape_bytes",
    "tfno_gated_delta_rule_workspace_bytes",
    "tfno_gated_delta_rule_step",
)

CONV_EXPORTS = EXPORTS[:8]   # the entry points with the (x, W, y, B, C_in, C_out, N, K, stream) signature
RECT_EXPORTS = EXPORTS[8:11]  # (x, W, y, B, C_in, C_out, N1, N2, K1, K2, stream)

_lib = None
_workspace = None     # the torch tensor currently registered as workspace (kept alive here)

# A small layer runs in a few microseconds on the device, so what a call costs on the host is its rate: torch, the entry
# points and the current-stream query are looked up once, and the workspace size of a shape (a function of the sizes alone)
# is kept for the most recent shapes (B 4, C 16, N 64: 8.4 -> 5.1 us per call, 3.2 of them the launch).
_torch = None
_raw_stream = None    # device index -> hipStream_t of the current stream


def _load_torch():
    global _torch, _raw_stream
    import torch
    _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
        lambda index: torch.cuda.current_stream(index).cuda_stream)
    _torch = torch
    return torch


@functools.lru_cache(maxsize=None)
def _entry(name: str):
    return getattr(lib(), name)


def _ask(query: str, *sizes) -> int:
    return _entry(query)(*sizes)


# The sizes of the most recent calls, for plain ints only: a mode count may be anything that ctypes takes for an int, and a 0-d
# array or tensor is not hashable, or compares by identity while its value changes (callers pick _ask for those).
_need = functools.lru_cache(maxsize=1024)(_ask)


def _check_c64(x, W, y):
    c64 = (_torch or _load_torch()).complex64
    for t, name in ((x, "x"), (W, "W"), (y, "y")):
        if t.dtype is not c64 or not t.is_contiguous() or not t.is_cuda:
            raise TypeError(f"{name} must be a contiguous complex64 device tensor")


def _check_real(x, W, y):
    torch = _torch or _load_torch()
    if x.dtype is not torch.float32 or y.dtype is not torch.float32 or W.dtype is not torch.complex64:
        raise TypeError("x, y must be float32 and W complex64")
    for t, name in ((x, "x"), (W, "W"), (y, "y")):
        if not t.is_contiguous() or not t.is_cuda:
            raise TypeError(f"{name} must be a contiguous device tensor")


def _launch(name: str, x, W, y, sizes, stream):
    if stream is None:
        stream = _raw_stream(x.device.index)
    st = _entry(name)(x.data_ptr(), W.data_ptr(), y.data_ptr(), *sizes, stream)
    if st != OK:
        raise TfnoError(st, name)
    return y


class _Strides(ctypes.Structure):
    _fields_ = [(n, ctypes.c_longlong) for n in ("batch", "token", "head")]


class _HeadNormDesc(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int) for n in ("dtype", "B", "T", "Hq", "Hk", "D", "R", "P", "interleaved")] +
                [("eps", ctypes.c_float), ("positions_batch", ctypes.c_longlong)] +
                [(n, _Strides) for n in ("q", "k", "q_out", "k_out", "dq", "dk")])


class _DeltaRuleDesc(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int) for n in ("dtype", "B", "T", "Hk", "Hv", "Dk", "Dv")] + [("scale", ctypes.c_float)] +
                [(n, _Strides) for n in ("q", "k", "v", "o", "g", "beta", "dq", "dk", "dv", "dg", "dbeta")])


class TfnoError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status})")


def lib() -> ctypes.CDLL:
    """Loads libtfno.so (built in-tree by ``python -m paper_2504_11681_amd.build``)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2504_11681_amd.build` "
                               "(there is no fallback path)")
        L = ctypes.CDLL(LIB_PATH)
        vp, ci = ctypes.c_void_p, ctypes.c_int
        for name in CONV_EXPORTS + ("tfno_spectral_conv1d_permode", "tfno_spectral_conv1d_real",
                                    "tfno_spectral_conv2d_noalloc"):
            fn = getattr(L, name)
            fn.restype = ci
            fn.argtypes = [vp, vp, vp, ci, ci, ci, ci, ci, vp]
        for name in RECT_EXPORTS + ("tfno_spectral_conv2d_strips",):
            fn = getattr(L, name)
            fn.restype = ci
            fn.argtypes = [vp, vp, vp] + [ci] * 7 + [vp]
        L.tfno_fno2d_real.restype = ci
        L.tfno_fno2d_real.argtypes = [vp, vp, vp] + [ci] * 7 + [vp]
        L.tfno_fno2d_real_workspace_bytes.restype = ctypes.c_size_t
        L.tfno_fno2d_real_workspace_bytes.argtypes = [ci] * 7
        L.tfno_fno1d_real.restype = ci
        L.tfno_fno1d_real.argtypes = [vp, vp, vp] + [ci] * 5 + [vp]
        L.tfno_fno1d_real_workspace_bytes.restype = ctypes.c_size_t
        L.tfno_fno1d_real_workspace_bytes.argtypes = [ci] * 5
        L.tfno_workspace_bytes.restype = ctypes.c_size_t
        L.tfno_workspace_bytes.argtypes = [ci] * 7
        L.tfno_workspace_bytes_2d.restype = ctypes.c_size_t
        L.tfno_workspace_bytes_2d.argtypes = [ci] * 8
        L.tfno_set_workspace.restype = ci
        L.tfno_set_workspace.argtypes = [vp, ctypes.c_size_t]
        L.tfno_status_string.restype = ctypes.c_char_p
        L.tfno_status_string.argtypes = [ci]
        L.tfno_version.restype = ci
        L.tfno_version.argtypes = []
        for name, pointers in (("tfno_head_norm_rope", 9), ("tfno_head_norm_rope_backward", 13), ("tfno_gated_delta_rule", 10),
                               ("tfno_gated_delta_rule_backward", 16)):
            fn = getattr(L, name)
            fn.restype = ci
            fn.argtypes = [vp] * (pointers + 2)      # the descriptor before them, the stream after
        L.tfno_gated_delta_rule_step.restype = ci
        L.tfno_gated_delta_rule_step.argtypes = [vp] * 8 + [ci, vp, vp]
        L.tfno_head_norm_rope_workspace_bytes.restype = ctypes.c_size_t
        L.tfno_head_norm_rope_workspace_bytes.argtypes = [ci]
        L.tfno_gated_delta_rule_tape_bytes.restype = ctypes.c_size_t
        L.tfno_gated_delta_rule_tape_bytes.argtypes = [vp]
        L.tfno_gated_delta_rule_workspace_bytes.restype = ctypes.c_size_t
        L.tfno_gated_delta_rule_workspace_bytes.argtypes = [vp, ci]
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().tfno_status_string(status).decode()


def version() -> int:
    return lib().tfno_version()


def workspace_bytes(dims: int, variant, B: int, C_in: int, C_out: int, N: int, K: int) -> int:
    """variant: 0 / False = fused entry point, 1 / True = staged twin, 2 = spectral_conv1d_pruned,
    3 = spectral_conv1d_fft_gemm, 4 = spectral_conv1d_gemm_ifft, 5 = spectral_conv1d_auto,
    6 = spectral_conv1d_permode."""
    return lib().tfno_workspace_bytes(dims, int(variant), B, C_in, C_out, N, K)


def workspace_bytes_2d(variant, B: int, C_in: int, C_out: int, N1: int, N2: int, K1: int, K2: int) -> int:
    """2-D entry points with per-axis sizes: variant 0 / False = spectral_conv2d_rect, 1 / True = its staged
    twin, 6 = spectral_conv2d_permode."""
    return lib().tfno_workspace_bytes_2d(int(variant), B, C_in, C_out, N1, N2, K1, K2)


def set_workspace(tensor) -> None:
    """Registers a torch device tensor (any dtype) as the library workspace; None clears it."""
    global _workspace
    if tensor is None:
        st = lib().tfno_set_workspace(None, 0)
    else:
        st = lib().tfno_set_workspace(tensor.data_ptr(), tensor.numel() * tensor.element_size())
    if st != OK:
        raise TfnoError(st, "tfno_set_workspace")
    _workspace = tensor


def ensure_workspace(nbytes: int, device) -> None:
    """Makes sure a registered workspace of at least nbytes exists (allocates with torch if not).

    The workspace is one buffer per process, shared by every stream.  Before a larger one replaces it the device is
    synchronised, so no kernel enqueued earlier on any stream still reads or writes the old buffer when torch frees
    it.  A HIP graph captured with the old buffer keeps the old address: growing the workspace invalidates such
    graphs (capture after the largest shape has been run once, or register a buffer of the final size up front with
    ``set_workspace``)."""
    import torch
    if nbytes == 0:
        return
    if _workspace is None or _workspace.numel() * _workspace.element_size() < nbytes or _workspace.device != device:
        if _workspace is not None:
            torch.cuda.synchronize(_workspace.device)
        set_workspace(torch.empty(nbytes, dtype=torch.uint8, device=device))


def _call(name: str, dims: int, variant: int, x, W, y, K: int, stream):
    _check_c64(x, W, y)
    xs, ws, ys = x.shape, W.shape, y.shape
    if len(xs) != 2 + dims or len(ys) != 2 + dims or len(ws) != 2:
        raise ValueError("x, y must be [B, C, N] (1-D) or [B, C, N, N] (2-D); W must be [C_in, C_out]")
    B, C_in, N = xs[0], xs[1], xs[2]
    C_out = ws[1]
    if ws[0] != C_in or ys[0] != B or ys[1] != C_out or ys[2:] != xs[2:] or xs[-1] != N:
        raise ValueError("inconsistent tensor shapes")
    need = (_need if type(K) is int else _ask)("tfno_workspace_bytes", dims, variant, B, C_in, C_out, N, K)
    if need:
        ensure_workspace(need, x.device)
    return _launch(name, x, W, y, (B, C_in, C_out, N, K), stream)


def spectral_conv1d(x, W, y, K: int, stream=None):
    return _call("tfno_spectral_conv1d", 1, 0, x, W, y, K, stream)


def spectral_conv2d(x, W, y, K: int, stream=None):
    return _call("tfno_spectral_conv2d", 2, 0, x, W, y, K, stream)


NOALLOC_SCRATCH_BYTES = 32 << 20     # TFNO_NOALLOC_SCRATCH_BYTES of the header


def spectral_conv2d_noalloc(x, W, y, K: int, stream=None):
    """tfno_spectral_conv2d with the library's own scratch array: allocates nothing and registers no workspace."""
    _check_c64(x, W, y)
    if x.dim() != 4 or y.dim() != 4 or W.dim() != 2 or x.shape[2] != x.shape[3]:
        raise ValueError("x, y must be [B, C, N, N]; W must be [C_in, C_out]")
    B, C_in, N = x.shape[0], x.shape[1], x.shape[2]
    C_out = W.shape[1]
    if W.shape[0] != C_in or tuple(y.shape) != (B, C_out, N, N):
        raise ValueError("inconsistent tensor shapes")
    return _launch("tfno_spectral_conv2d_noalloc", x, W, y, (B, C_in, C_out, N, K), stream)


def spectral_conv1d_staged(x, W, y, K: int, stream=None):
    return _call("tfno_spectral_conv1d_staged", 1, 1, x, W, y, K, stream)


def spectral_conv2d_staged(x, W, y, K: int, stream=None):
    return _call("tfno_spectral_conv2d_staged", 2, 1, x, W, y, K, stream)


def spectral_conv1d_pruned(x, W, y, K: int, stream=None):
    return _call("tfno_spectral_conv1d_pruned", 1, 2, x, W, y, K, stream)


def spectral_conv1d_fft_gemm(x, W, y, K: int, stream=None):
    return _call("tfno_spectral_conv1d_fft_gemm", 1, 3, x, W, y, K, stream)


def spectral_conv1d_gemm_ifft(x, W, y, K: int, stream=None):
    return _call("tfno_spectral_conv1d_gemm_ifft", 1, 4, x, W, y, K, stream)


def spectral_conv1d_auto(x, W, y, K: int, stream=None):
    return _call("tfno_spectral_conv1d_auto", 1, 5, x, W, y, K, stream)


def _call_rect(name: str, variant: int, x, W, y, K1: int, K2: int, stream):
    _check_c64(x, W, y)
    xs, ws, ys = x.shape, W.shape, y.shape
    if len(xs) != 4 or len(ys) != 4 or len(ws) != 2:
        raise ValueError("x, y must be [B, C, N1, N2]; W must be [C_in, C_out]")
    B, C_in, N1, N2 = xs
    C_out = ws[1]
    if ws[0] != C_in or ys[0] != B or ys[1] != C_out or ys[2:] != xs[2:]:
        raise ValueError("inconsistent tensor shapes")
    need = (_need if type(K1) is type(K2) is int else _ask)("tfno_workspace_bytes_2d", variant, B, C_in, C_out, N1, N2, K1, K2)
    if need:
        ensure_workspace(need, x.device)
    return _launch(name, x, W, y, (B, C_in, C_out, N1, N2, K1, K2), stream)


def spectral_conv2d_rect(x, W, y, K1: int, K2: int, stream=None):
    return _call_rect("tfno_spectral_conv2d_rect", 0, x, W, y, K1, K2, stream)


def spectral_conv2d_rect_staged(x, W, y, K1: int, K2: int, stream=None):
    return _call_rect("tfno_spectral_conv2d_rect_staged", 1, x, W, y, K1, K2, stream)


def spectral_conv2d_strips(x, W, y, K1: int, K2: int, stream=None):
    """The paper's 2-D pipeline on request (first-axis FFT, fused 1-D kernel on the retained rows, first-axis iFFT)."""
    return _call_rect("tfno_spectral_conv2d_strips", 7, x, W, y, K1, K2, stream)


def _call_permode(name: str, dims: int, x, W, y, stream):
    _check_c64(x, W, y)
    xs, ws, ys = x.shape, W.shape, y.shape
    if len(xs) != 2 + dims or len(ys) != 2 + dims or len(ws) != 2 + dims:
        raise ValueError("x, y must be [B, C, spatial...]; W must be [C_in, C_out, modes...]")
    B, C_in = xs[0], xs[1]
    C_out = ws[1]
    if ws[0] != C_in or ys[0] != B or ys[1] != C_out or ys[2:] != xs[2:]:
        raise ValueError("inconsistent tensor shapes")
    if dims == 1:
        sizes = (B, C_in, C_out, xs[2], ws[2])
        need = _need("tfno_workspace_bytes", 1, 6, *sizes)
    else:
        sizes = (B, C_in, C_out, xs[2], xs[3], ws[2], ws[3])
        need = _need("tfno_workspace_bytes_2d", 6, *sizes)
    if need:
        ensure_workspace(need, x.device)
    return _launch(name, x, W, y, sizes, stream)


def spectral_conv1d_permode(x, W, y, stream=None):
    """W: [C_in, C_out, K], an own weight matrix per retained mode."""
    return _call_permode("tfno_spectral_conv1d_permode", 1, x, W, y, stream)


def spectral_conv2d_permode(x, W, y, stream=None):
    """W: [C_in, C_out, K1, K2]."""
    return _call_permode("tfno_spectral_conv2d_permode", 2, x, W, y, stream)


def spectral_conv1d_real(x, W, y, K: int, stream=None):
    """Real-valued layer: x [B, C_in, N] and y [B, C_out, N] float32 device tensors, W [C_in, C_out] complex64."""
    _check_real(x, W, y)
    xs, ws, ys = x.shape, W.shape, y.shape
    if len(xs) != 3 or len(ys) != 3 or len(ws) != 2:
        raise ValueError("x, y must be [B, C, N]; W must be [C_in, C_out]")
    B, C_in, N = xs
    C_out = ws[1]
    if ws[0] != C_in or ys[0] != B or ys[1] != C_out or ys[2] != N:
        raise ValueError("inconsistent tensor shapes")
    return _launch("tfno_spectral_conv1d_real", x, W, y, (B, C_in, C_out, N, K), stream)


def fno2d_real(x, W, y, stream=None):
    """The 2-D Fourier layer of FNO models on real fields: x [B, C_in, N1, N2] and y [B, C_out, N1, N2] float32,
    W [C_in, C_out, 2*M1, M2] complex64 (first-axis frequencies -M1..M1-1, last-axis 0..M2-1)."""
    _check_real(x, W, y)
    xs, ws, ys = x.shape, W.shape, y.shape
    if len(xs) != 4 or len(ys) != 4 or len(ws) != 4 or ws[2] % 2:
        raise ValueError("x, y must be [B, C, N1, N2]; W must be [C_in, C_out, 2*M1, M2]")
    B, C_in, N1, N2 = xs
    C_out = ws[1]
    if ws[0] != C_in or ys[0] != B or ys[1] != C_out or ys[2:] != xs[2:]:
        raise ValueError("inconsistent tensor shapes")
    sizes = (B, C_in, C_out, N1, N2, ws[2] // 2, ws[3])
    need = _need("tfno_fno2d_real_workspace_bytes", *sizes)
    if need:
        ensure_workspace(need, x.device)
    return _launch("tfno_fno2d_real", x, W, y, sizes, stream)


def fno1d_real(x, W, y, stream=None):
    """The 1-D Fourier layer of FNO models on real fields: x [B, C_in, N], y [B, C_out, N] float32,
    W [C_in, C_out, M] complex64 (one matrix per mode 0..M-1)."""
    _check_real(x, W, y)
    xs, ws, ys = x.shape, W.shape, y.shape
    if len(xs) != 3 or len(ys) != 3 or len(ws) != 3:
        raise ValueError("x, y must be [B, C, N]; W must be [C_in, C_out, M]")
    B, C_in, N = xs
    C_out = ws[1]
    if ws[0] != C_in or ys[0] != B or ys[1] != C_out or ys[2] != N:
        raise ValueError("inconsistent tensor shapes")
    sizes = (B, C_in, C_out, N, ws[2])
    need = _need("tfno_fno1d_real_workspace_bytes", *sizes)
    if need:
        ensure_workspace(need, x.device)
    return _launch("tfno_fno1d_real", x, W, y, sizes, stream)


# ---------------------------------------------------------------- operators along time

def _element_type(dtype) -> int:
    torch = _torch or _load_torch()
    if dtype is torch.bfloat16:
        return 1
    if dtype is torch.float32:
        return 0
    raise TypeError("q, k and v must be float32 or bfloat16")


def _tensors(first, others, **named):
    """Checks what the operators along time take: device tensors of the type of `first` (others) or of the type given (named; None passes),
    whose last axis is contiguous."""
    for name, t in others.items():
        if t.dtype is not first.dtype:
            raise TypeError(f"{name} must have the type of q")
    checks = list(others.items())
    for name, (t, dtype) in named.items():
        if t is not None:
            if t.dtype is not dtype:
                raise TypeError(f"{name} must be {dtype}")
            checks.append((name, t))
    for name, t in checks:
        if not t.is_cuda or t.device != first.device:
            raise TypeError(f"{name} must be a tensor on the device of q")


def _layout(t):
    return None if t is None else (t.shape, t.stride())


def _strides4(name, layout, shape):
    """Strides of a [B, T, H, D] tensor with its last axis contiguous."""
    if tuple(layout[0]) != shape:
        raise ValueError(f"{name} must be {list(shape)}, not {list(layout[0])}")
    if shape[3] > 1 and layout[1][3] != 1:
        raise ValueError(f"the last axis of {name} must be contiguous")
    return _Strides(*layout[1][:3])


def _contiguous(**tensors):
    for name, t in tensors.items():
        if t is not None and not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")


def _ptr(t):
    return None if t is None else t.data_ptr()


@functools.lru_cache(maxsize=1024)
def _head_norm_desc(dtype, q, k, q_out, k_out, dq, dk, positions, wq, wk, dwq, dwk, cos, sin, eps, interleaved):
    if len(q[0]) != 4 or len(k[0]) != 4 or q[0][:2] != k[0][:2] or q[0][3] != k[0][3]:
        raise ValueError("q and k must be [B, T, Hq, D] and [B, T, Hk, D]")
    B, T, Hq, D = q[0]
    Hk = k[0][2]
    for name, w in (("wq", wq), ("wk", wk), ("dwq", dwq), ("dwk", dwk)):
        if w is not None and tuple(w[0]) != (D,):
            raise ValueError(f"{name} must be [D]")
    if (cos is None) != (sin is None) or (cos is not None and (len(cos[0]) != 2 or cos[0] != sin[0])):
        raise ValueError("cos and sin must both be [P, R / 2], or both None")
    P, R = (0, 0) if cos is None else (cos[0][0], 2 * cos[0][1])
    d = _HeadNormDesc(_element_type(dtype), B, T, Hq, Hk, D, R, P, int(interleaved), eps, 0)
    if positions is not None:
        if tuple(positions[0]) != (B, T) or (T > 1 and positions[1][1] != 1):
            raise ValueError("positions must be [B, T] with contiguous rows")
        d.positions_batch = positions[1][0]
    for name, t, H in (("q", q, Hq), ("k", k, Hk), ("q_out", q_out, Hq), ("k_out", k_out, Hk), ("dq", dq, Hq), ("dk", dk, Hk)):
        if t is not None:
            setattr(d, name, _strides4(name, t, (B, T, H, D)))
    return d, ctypes.addressof(d)


def head_norm_rope(q, k, wq, wk, cos, sin, q_out, k_out, positions=None, eps: float = 1e-6, interleaved: bool = False, stream=None):
    """Norm of queries and keys for each head with the rotation by position: q [B, T, Hq, D] and k [B, T, Hk, D] (float32 or bfloat16, any
    strides with the last axis contiguous) into q_out and k_out, which may be q and k themselves.  wq, wk: float32 [D] or None (ones);
    cos, sin: float32 [P, R / 2] or None (no rotation); positions: int32 [B, T] or None (0 .. T - 1)."""
    f32, i32 = (_torch or _load_torch()).float32, _torch.int32
    _tensors(q, {"q": q, "k": k, "q_out": q_out, "k_out": k_out}, wq=(wq, f32), wk=(wk, f32), cos=(cos, f32), sin=(sin, f32), positions=(positions, i32))
    _contiguous(wq=wq, wk=wk, cos=cos, sin=sin)
    d = _head_norm_desc(q.dtype, _layout(q), _layout(k), _layout(q_out), _layout(k_out), None, None, _layout(positions), _layout(wq), _layout(wk),
                        None, None, _layout(cos), _layout(sin), eps, interleaved)
    st = _entry("tfno_head_norm_rope")(d[1], q.data_ptr(), k.data_ptr(), _ptr(wq), _ptr(wk), _ptr(cos), _ptr(sin), _ptr(positions),
                                       q_out.data_ptr(), k_out.data_ptr(), _raw_stream(q.device.index) if stream is None else stream)
    if st != OK:
        raise TfnoError(st, "tfno_head_norm_rope")
    return q_out, k_out


def head_norm_rope_backward(q, k, wq, wk, cos, sin, dq_out, dk_out, dq, dk, dwq=None, dwk=None, positions=None, eps: float = 1e-6,
                            interleaved: bool = False, stream=None):
    """Gradients dq, dk and, where given, dwq, dwk (float32 [D]) of head_norm_rope from those of its results, dq_out and dk_out."""
    f32, i32 = (_torch or _load_torch()).float32, _torch.int32
    _tensors(q, {"q": q, "k": k, "dq_out": dq_out, "dk_out": dk_out, "dq": dq, "dk": dk}, wq=(wq, f32), wk=(wk, f32), cos=(cos, f32), sin=(sin, f32),
             positions=(positions, i32), dwq=(dwq, f32), dwk=(dwk, f32))
    _contiguous(wq=wq, wk=wk, cos=cos, sin=sin, dwq=dwq, dwk=dwk)
    d = _head_norm_desc(q.dtype, _layout(q), _layout(k), _layout(dq_out), _layout(dk_out), _layout(dq), _layout(dk), _layout(positions), _layout(wq),
                        _layout(wk), _layout(dwq), _layout(dwk), _layout(cos), _layout(sin), eps, interleaved)
    ensure_workspace(_need("tfno_head_norm_rope_workspace_bytes", d[0].D), q.device)
    st = _entry("tfno_head_norm_rope_backward")(d[1], q.data_ptr(), k.data_ptr(), _ptr(wq), _ptr(wk), _ptr(cos), _ptr(sin), _ptr(positions),
                                                dq_out.data_ptr(), dk_out.data_ptr(), dq.data_ptr(), dk.data_ptr(), _ptr(dwq), _ptr(dwk),
                                                _raw_stream(q.device.index) if stream is None else stream)
    if st != OK:
        raise TfnoError(st, "tfno_head_norm_rope_backward")
    return dq, dk


@functools.lru_cache(maxsize=1024)
def _rule_desc(dtype, q, k, v, o, g, beta, dq, dk, dv, dg, dbeta, scale):
    """The descriptor of a call, its address, the shape of its states, and the bytes of its tape and workspaces."""
    if len(q[0]) != 4 or len(v[0]) != 4 or q[0][:2] != v[0][:2]:
        raise ValueError("q, k must be [B, T, Hk, Dk] and v [B, T, Hv, Dv]")
    B, T, Hk, Dk = q[0]
    Hv, Dv = v[0][2:]
    d = _DeltaRuleDesc(_element_type(dtype), B, T, Hk, Hv, Dk, Dv, Dk ** -0.5 if scale is None else scale)
    for name, t, shape in (("q", q, (Hk, Dk)), ("k", k, (Hk, Dk)), ("v", v, (Hv, Dv)), ("o", o, (Hv, Dv)), ("dq", dq, (Hk, Dk)), ("dk", dk, (Hk, Dk)),
                           ("dv", dv, (Hv, Dv))):
        if t is not None:
            setattr(d, name, _strides4(name, t, (B, T, *shape)))
    for name, t in (("g", g), ("beta", beta), ("dg", dg), ("dbeta", dbeta)):
        if t is not None:
            if tuple(t[0]) != (B, T, Hv):
                raise ValueError(f"{name} must be [B, T, Hv]")
            setattr(d, name, _Strides(*t[1]))
    at = ctypes.addressof(d)
    ask = _entry("tfno_gated_delta_rule_workspace_bytes")
    return d, at, (B, Hv, Dk, Dv), _entry("tfno_gated_delta_rule_tape_bytes")(at), ask(at, 0), ask(at, 1)


def _check_states(shape, B, tape, need, lengths, **states):
    for name, t in states.items():
        if t is not None and (tuple(t.shape) != shape or not t.is_contiguous()):
            raise ValueError(f"{name} must be a contiguous {list(shape)}")
    if lengths is not None and (tuple(lengths.shape) != (B,) or not lengths.is_contiguous()):
        raise ValueError("lengths must be a contiguous [B]")
    if tape is not None and (not tape.is_contiguous() or tape.numel() * tape.element_size() < need):
        raise ValueError(f"the tape must be contiguous and hold {need} bytes")


def gated_delta_rule_tape(q, v):
    """A tape for gated_delta_rule and gated_delta_rule_backward on tensors of the sizes of q [B, T, Hk, Dk] and v [B, T, Hv, Dv]."""
    torch = _torch or _load_torch()
    d = _rule_desc(q.dtype, _layout(q), _layout(q), _layout(v), None, None, None, None, None, None, None, None, None)
    return torch.empty(d[3], dtype=torch.uint8, device=q.device)


def gated_delta_rule(q, k, v, g, beta, o, scale=None, initial_state=None, final_state=None, lengths=None, tape=None, stream=None):
    """The gated delta rule over whole sequences: q, k [B, T, Hk, Dk], v, o [B, T, Hv, Dv] (float32 or bfloat16, any strides with the last axis
    contiguous), g (log decay, or None) and beta float32 [B, T, Hv], states float32 [B, Hv, Dk, Dv], lengths int32 [B].  scale is Dk ** -0.5
    where it is not given.  With a tape (gated_delta_rule_tape) the gradient can be taken afterwards."""
    f32, i32 = (_torch or _load_torch()).float32, _torch.int32
    _tensors(q, {"q": q, "k": k, "v": v, "o": o}, g=(g, f32), beta=(beta, f32), initial_state=(initial_state, f32), final_state=(final_state, f32),
             lengths=(lengths, i32), tape=(tape, _torch.uint8))
    d = _rule_desc(q.dtype, _layout(q), _layout(k), _layout(v), _layout(o), _layout(g), _layout(beta), None, None, None, None, None, scale)
    _check_states(d[2], d[2][0], tape, d[3], lengths, initial_state=initial_state, final_state=final_state)
    if tape is None:
        ensure_workspace(d[4], q.device)
    st = _entry("tfno_gated_delta_rule")(d[1], q.data_ptr(), k.data_ptr(), v.data_ptr(), _ptr(g), beta.data_ptr(), _ptr(lengths), _ptr(initial_state),
                                         o.data_ptr(), _ptr(final_state), _ptr(tape), _raw_stream(q.device.index) if stream is None else stream)
    if st != OK:
        raise TfnoError(st, "tfno_gated_delta_rule")
    return o


def gated_delta_rule_backward(q, k, v, g, beta, d_o, dq, dk, dv, dg, dbeta, tape, scale=None, initial_state=None, d_final_state=None,
                              d_initial_state=None, lengths=None, stream=None):
    """Gradients of gated_delta_rule with the same inputs, from its tape and the gradients d_o of o and d_final_state of the final state
    (None: zeros).  dg and d_initial_state may be None."""
    f32, i32 = (_torch or _load_torch()).float32, _torch.int32
    _tensors(q, {"q": q, "k": k, "v": v, "d_o": d_o, "dq": dq, "dk": dk, "dv": dv}, g=(g, f32), beta=(beta, f32), dg=(dg, f32), dbeta=(dbeta, f32),
             initial_state=(initial_state, f32), d_final_state=(d_final_state, f32), d_initial_state=(d_initial_state, f32), lengths=(lengths, i32),
             tape=(tape, _torch.uint8))
    d = _rule_desc(q.dtype, _layout(q), _layout(k), _layout(v), _layout(d_o), _layout(g), _layout(beta), _layout(dq), _layout(dk), _layout(dv),
                   _layout(dg), _layout(dbeta), scale)
    _check_states(d[2], d[2][0], tape, d[3], lengths, initial_state=initial_state, d_final_state=d_final_state, d_initial_state=d_initial_state)
    ensure_workspace(d[5], q.device)
    st = _entry("tfno_gated_delta_rule_backward")(
        d[1], q.data_ptr(), k.data_ptr(), v.data_ptr(), _ptr(g), beta.data_ptr(), _ptr(lengths), _ptr(initial_state), tape.data_ptr(), d_o.data_ptr(),
        _ptr(d_final_state), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), _ptr(dg), dbeta.data_ptr(), _ptr(d_initial_state),
        _raw_stream(q.device.index) if stream is None else stream)
    if st != OK:
        raise TfnoError(st, "tfno_gated_delta_rule_backward")
    return dq, dk, dv, dg, dbeta


@functools.lru_cache(maxsize=1024)
def _step_desc(dtype, q, k, v, o, g, beta, states, scale):
    if len(q[0]) != 3 or len(v[0]) != 3 or q[0][0] != v[0][0]:
        raise ValueError("q, k must be [B, Hk, Dk] and v [B, Hv, Dv]")
    B, Hk, Dk = q[0]
    Hv, Dv = v[0][1:]
    if len(states) != 4 or tuple(states[1:]) != (Hv, Dk, Dv):
        raise ValueError("states must be [pool, Hv, Dk, Dv]")
    d = _DeltaRuleDesc(_element_type(dtype), B, 1, Hk, Hv, Dk, Dv, Dk ** -0.5 if scale is None else scale)
    for name, t, shape in (("q", q, (Hk, Dk)), ("k", k, (Hk, Dk)), ("v", v, (Hv, Dv)), ("o", o, (Hv, Dv))):
        s = t[1]
        setattr(d, name, _strides4(name, ((B, 1, *t[0][1:]) if t[0][0] == B else t[0], (s[0], 0, s[1], s[2])), (B, 1, *shape)))
    for name, t in (("g", g), ("beta", beta)):
        if t is not None:
            if tuple(t[0]) != (B, Hv):
                raise ValueError(f"{name} must be [B, Hv]")
            setattr(d, name, _Strides(t[1][0], 0, t[1][1]))
    return d, ctypes.addressof(d)


def gated_delta_rule_step(q, k, v, g, beta, states, o, slots=None, scale=None, stream=None):
    """One token of the gated delta rule: q, k [B, Hk, Dk], v, o [B, Hv, Dv], g (or None) and beta float32 [B, Hv]; the states float32
    [pool, Hv, Dk, Dv] of the slots int32 [B] (None: 0 .. B - 1; negative: no sequence) are advanced in place."""
    f32, i32 = (_torch or _load_torch()).float32, _torch.int32
    _tensors(q, {"q": q, "k": k, "v": v, "o": o}, g=(g, f32), beta=(beta, f32), states=(states, f32), slots=(slots, i32))
    d = _step_desc(q.dtype, _layout(q), _layout(k), _layout(v), _layout(o), _layout(g), _layout(beta), states.shape, scale)
    _contiguous(states=states, slots=slots)
    if slots is not None and tuple(slots.shape) != (q.shape[0],):
        raise ValueError("slots must be [B]")
    st = _entry("tfno_gated_delta_rule_step")(d[1], q.data_ptr(), k.data_ptr(), v.data_ptr(), _ptr(g), beta.data_ptr(), states.data_ptr(), _ptr(slots),
                                              states.shape[0], o.data_ptr(), _raw_stream(q.device.index) if stream is None else stream)
    if st != OK:
        raise TfnoError(st, "tfno_gated_delta_rule_step")
    return o
