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
    "tfno_gated_recurrence",
    "tfno_gated_recurrence_backward",
    "tfno_gated_recurrence_tape_bytes",
    "tfno_gated_recurrence_workspace_bytes",
    "tfno_gated_recurrence_step",
    "tfno_block_norm",
    "tfno_block_norm_backward",
    "tfno_block_norm_workspace_bytes",
    "tfno_clip_grad_norm",
    "tfno_clip_grad_norm_workspace_bytes",
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


class _RecurrenceDesc(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int) for n in ("dtype", "B", "T", "C", "normalise")] +
                [(n, _Strides) for n in ("x", "gate", "input_gate", "y", "dx", "dgate", "dinput_gate")])


class _BlockNormDesc(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int) for n in ("dtype", "residual_dtype", "B", "T", "C", "gate_kind", "activation", "norm_after")] +
                [("residual_scale", ctypes.c_float), ("eps", ctypes.c_float)] +
                [(n, _Strides) for n in ("y", "r", "gate", "r_out", "n_out", "dy", "dr", "dgate")])


class _Tensor(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("elements", ctypes.c_longlong), ("dtype", ctypes.c_int)]


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
        for name, pointers in (("tfno_gated_recurrence", 9), ("tfno_gated_recurrence_backward", 13), ("tfno_block_norm", 8),
                               ("tfno_block_norm_backward", 13)):
            fn = getattr(L, name)
            fn.restype = ci
            fn.argtypes = [vp] * (pointers + 2)      # the descriptor before them, the stream after
        L.tfno_gated_recurrence_step.restype = ci
        L.tfno_gated_recurrence_step.argtypes = [vp] * 7 + [ci, vp, vp]
        L.tfno_clip_grad_norm.restype = ci
        L.tfno_clip_grad_norm.argtypes = [vp, ci, ctypes.c_double, vp, vp]
        for name, arguments in (("tfno_gated_recurrence_tape_bytes", [vp]), ("tfno_gated_recurrence_workspace_bytes", [vp, ci]),
                                ("tfno_block_norm_workspace_bytes", [vp]), ("tfno_clip_grad_norm_workspace_bytes", [ci])):
            fn = getattr(L, name)
            fn.restype = ctypes.c_size_t
            fn.argtypes = arguments
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
#
# A call's descriptor and all checks of its arguments depend on types, devices, shapes and strides alone.  They are made once for each such
# combination (_plan) and looked up afterwards: what a call costs on the host is its rate for one token.  The combination's key and the call
# itself are made in C++ (csrc/marshal.cpp).

_plans = {}
_marshal = None


def _load_marshal():
    global _marshal
    lib()
    if _torch is None:
        _load_torch()
    try:
        from . import _marshal as m
    except ImportError as e:
        raise RuntimeError("_marshal.so is missing or of another torch: build it with `python -m paper_2504_11681_amd.build` "
                           "(there is no fallback path)") from e
    m.open(LIB_PATH)
    _marshal = m
    return m


def _of(t):
    """What a plan depends on of a tensor."""
    return None if t is None else (t.dtype, t.get_device(), t.shape, t.stride())


def _plan(key, make, tensors, *args):
    if len(_plans) >= 4096:
        _plans.clear()
    plan = _plans[key] = make(*map(_of, tensors), *args)
    return plan


def _element_type(dtype, what="q, k and v") -> int:
    torch = _torch or _load_torch()
    if dtype is torch.bfloat16:
        return 1
    if dtype is torch.float32:
        return 0
    raise TypeError(f"{what} must be float32 or bfloat16")


def _check_types(first, same, f32=(), i32=(), u8=(), what="q"):
    """Device tensors on one device: `same` of the type of the first one, the others of the types named; each given as (name, _of(tensor))."""
    torch = _torch or _load_torch()
    _element_type(first[0], "q, k and v" if what == "q" else what)
    for dtype, tensors in ((first[0], same), (torch.float32, f32), (torch.int32, i32), (torch.uint8, u8)):
        for name, t in tensors:
            if t is None:
                continue
            if t[0] is not dtype:
                raise TypeError(f"{name} must be {dtype}")
            if t[1] < 0 or t[1] != first[1]:
                raise TypeError(f"{name} must be a tensor on the device of {what}")


def _strides4(name, t, shape):
    """Strides of a [B, T, H, D] tensor with its last axis contiguous."""
    if tuple(t[2]) != shape:
        raise ValueError(f"{name} must be {list(shape)}, not {list(t[2])}")
    if shape[3] > 1 and t[3][3] != 1:
        raise ValueError(f"the last axis of {name} must be contiguous")
    return _Strides(*t[3][:3])


def _check_contiguous(shape, *tensors):
    for name, t in tensors:
        if t is None:
            continue
        if tuple(t[2]) != tuple(shape):
            raise ValueError(f"{name} must be {list(shape)}, not {list(t[2])}")
        step = 1
        for size, stride in zip(reversed(t[2]), reversed(t[3])):
            if size > 1 and stride != step:
                raise ValueError(f"{name} must be contiguous")
            step *= size


def _head_norm_plan(q, k, q_out, k_out, dq, dk, positions, wq, wk, dwq, dwk, cos, sin, eps, interleaved):
    names = (("q", q), ("k", k), ("q_out", q_out), ("k_out", k_out), ("dq", dq), ("dk", dk))
    _check_types(q, names, f32=(("wq", wq), ("wk", wk), ("dwq", dwq), ("dwk", dwk), ("cos", cos), ("sin", sin)), i32=(("positions", positions),))
    if len(q[2]) != 4 or len(k[2]) != 4 or q[2][:2] != k[2][:2] or q[2][3] != k[2][3]:
        raise ValueError("q and k must be [B, T, Hq, D] and [B, T, Hk, D]")
    B, T, Hq, D = q[2]
    Hk = k[2][2]
    _check_contiguous((D,), ("wq", wq), ("wk", wk), ("dwq", dwq), ("dwk", dwk))
    if (cos is None) != (sin is None) or (cos is not None and (len(cos[2]) != 2 or cos[2] != sin[2])):
        raise ValueError("cos and sin must both be [P, R / 2], or both None")
    P, R = (0, 0) if cos is None else (cos[2][0], 2 * cos[2][1])
    _check_contiguous((P, R // 2), ("cos", cos), ("sin", sin))
    d = _HeadNormDesc(_element_type(q[0]), B, T, Hq, Hk, D, R, P, int(interleaved), eps, 0)
    if positions is not None:
        if tuple(positions[2]) != (B, T) or (T > 1 and positions[3][1] != 1):
            raise ValueError("positions must be [B, T] with contiguous rows")
        d.positions_batch = positions[3][0]
    for (name, t), H in zip(names, (Hq, Hk) * 3):
        if t is not None:
            setattr(d, name, _strides4(name, t, (B, T, H, D)))
    need = 0 if dwq is None and dwk is None else _entry("tfno_head_norm_rope_workspace_bytes")(D)
    return ctypes.addressof(d), need, q[1], d


def head_norm_rope(q, k, wq, wk, cos, sin, q_out, k_out, positions=None, eps: float = 1e-6, interleaved: bool = False, stream=None):
    """Norm of queries and keys for each head with the rotation by position: q [B, T, Hq, D] and k [B, T, Hk, D] (float32 or bfloat16, any
    strides with the last axis contiguous) into q_out and k_out, which may be q and k themselves.  wq, wk: float32 [D] or None (ones);
    cos, sin: float32 [P, R / 2] or None (no rotation); positions: int32 [B, T] or None (0 .. T - 1)."""
    m = _marshal or _load_marshal()
    tensors = (q, k, q_out, k_out, None, None, positions, wq, wk, None, None, cos, sin)
    key = (m.key(*tensors), eps := float(eps), interleaved := bool(interleaved))
    plan = _plans.get(key) or _plan(key, _head_norm_plan, tensors, eps, interleaved)
    st = m.tfno_head_norm_rope(plan[0], q, k, wq, wk, cos, sin, positions, q_out, k_out, _raw_stream(plan[2]) if stream is None else stream)
    if st != OK:
        raise TfnoError(st, "tfno_head_norm_rope")
    return q_out, k_out


def head_norm_rope_backward(q, k, wq, wk, cos, sin, dq_out, dk_out, dq, dk, dwq=None, dwk=None, positions=None, eps: float = 1e-6,
                            interleaved: bool = False, stream=None):
    """Gradients dq, dk and, where given, dwq, dwk (float32 [D]) of head_norm_rope from those of its results, dq_out and dk_out."""
    m = _marshal or _load_marshal()
    tensors = (q, k, dq_out, dk_out, dq, dk, positions, wq, wk, dwq, dwk, cos, sin)
    key = (m.key(*tensors), eps := float(eps), interleaved := bool(interleaved))
    plan = _plans.get(key) or _plan(key, _head_norm_plan, tensors, eps, interleaved)
    ensure_workspace(plan[1], q.device)
    st = m.tfno_head_norm_rope_backward(plan[0], q, k, wq, wk, cos, sin, positions, dq_out, dk_out, dq, dk, dwq, dwk,
                                        _raw_stream(plan[2]) if stream is None else stream)
    if st != OK:
        raise TfnoError(st, "tfno_head_norm_rope_backward")
    return dq, dk


def _rule_plan(q, k, v, o, g, beta, dq, dk, dv, dg, dbeta, lengths, tape, initial, final, other, scale):
    names = (("q", q), ("k", k), ("v", v), ("o", o), ("dq", dq), ("dk", dk), ("dv", dv))
    gates = (("g", g), ("beta", beta), ("dg", dg), ("dbeta", dbeta))
    states = (("the initial state", initial), ("the final state or its gradient", final), ("the gradient of the initial state", other))
    _check_types(q, names, f32=gates + states, i32=(("lengths", lengths),), u8=(("the tape", tape),))
    if len(q[2]) != 4 or len(v[2]) != 4 or q[2][:2] != v[2][:2]:
        raise ValueError("q, k must be [B, T, Hk, Dk] and v [B, T, Hv, Dv]")
    B, T, Hk, Dk = q[2]
    Hv, Dv = v[2][2:]
    d = _DeltaRuleDesc(_element_type(q[0]), B, T, Hk, Hv, Dk, Dv, Dk ** -0.5 if scale is None else scale)
    for (name, t), shape in zip(names, ((Hk, Dk), (Hk, Dk), (Hv, Dv), (Hv, Dv), (Hk, Dk), (Hk, Dk), (Hv, Dv))):
        if t is not None:
            setattr(d, name, _strides4(name, t, (B, T, *shape)))
    for name, t in gates:
        if t is not None:
            if tuple(t[2]) != (B, T, Hv):
                raise ValueError(f"{name} must be [B, T, Hv]")
            setattr(d, name, _Strides(*t[3]))
    _check_contiguous((B, Hv, Dk, Dv), *states)
    _check_contiguous((B,), ("lengths", lengths))
    at = ctypes.addressof(d)
    need = _entry("tfno_gated_delta_rule_tape_bytes")(at)
    if tape is not None and (len(tape[2]) != 1 or tape[3][0] != 1 or tape[2][0] < need):
        raise ValueError(f"the tape must be contiguous and hold {need} bytes")
    ask = _entry("tfno_gated_delta_rule_workspace_bytes")
    return at, need, ask(at, 0), ask(at, 1), q[1], d


def gated_delta_rule_tape(q, v):
    """A tape for gated_delta_rule and gated_delta_rule_backward on tensors of the sizes of q [B, T, Hk, Dk] and v [B, T, Hv, Dv]."""
    torch = _torch or _load_torch()
    m = _marshal or _load_marshal()
    key = ("tape", m.key(q, v))
    plan = _plans.get(key) or _plan(key, _rule_plan, (q, q, v, *(None,) * 13), None)
    return torch.empty(plan[1], dtype=torch.uint8, device=q.device)


def gated_delta_rule(q, k, v, g, beta, o, scale=None, initial_state=None, final_state=None, lengths=None, tape=None, stream=None):
    """The gated delta rule over whole sequences: q, k [B, T, Hk, Dk], v, o [B, T, Hv, Dv] (float32 or bfloat16, any strides with the last axis
    contiguous), g (log decay, or None) and beta float32 [B, T, Hv], states float32 [B, Hv, Dk, Dv], lengths int32 [B].  scale is Dk ** -0.5
    where it is not given.  With a tape (gated_delta_rule_tape) the gradient can be taken afterwards."""
    m = _marshal or _load_marshal()
    tensors = (q, k, v, o, g, beta, None, None, None, None, None, lengths, tape, initial_state, final_state, None)
    key = ("rule", m.key(*tensors), scale := None if scale is None else float(scale))
    plan = _plans.get(key) or _plan(key, _rule_plan, tensors, scale)
    if tape is None:
        ensure_workspace(plan[2], q.device)
    st = m.tfno_gated_delta_rule(plan[0], q, k, v, g, beta, lengths, initial_state, o, final_state, tape,
                                 _raw_stream(plan[4]) if stream is None else stream)
    if st != OK:
        raise TfnoError(st, "tfno_gated_delta_rule")
    return o


def gated_delta_rule_backward(q, k, v, g, beta, d_o, dq, dk, dv, dg, dbeta, tape, scale=None, initial_state=None, d_final_state=None,
                              d_initial_state=None, lengths=None, stream=None):
    """Gradients of gated_delta_rule with the same inputs, from its tape and the gradients d_o of o and d_final_state of the final state
    (None: zeros).  dg and d_initial_state may be None."""
    m = _marshal or _load_marshal()
    tensors = (q, k, v, d_o, g, beta, dq, dk, dv, dg, dbeta, lengths, tape, initial_state, d_final_state, d_initial_state)
    key = ("rule", m.key(*tensors), scale := None if scale is None else float(scale))
    plan = _plans.get(key) or _plan(key, _rule_plan, tensors, scale)
    ensure_workspace(plan[3], q.device)
    st = m.tfno_gated_delta_rule_backward(plan[0], q, k, v, g, beta, lengths, initial_state, tape, d_o, d_final_state, dq, dk, dv, dg, dbeta,
                                          d_initial_state, _raw_stream(plan[4]) if stream is None else stream)
    if st != OK:
        raise TfnoError(st, "tfno_gated_delta_rule_backward")
    return dq, dk, dv, dg, dbeta


def _step_plan(q, k, v, o, g, beta, states, slots, scale):
    names = (("q", q), ("k", k), ("v", v), ("o", o))
    _check_types(q, names, f32=(("g", g), ("beta", beta), ("states", states)), i32=(("slots", slots),))
    if len(q[2]) != 3 or len(v[2]) != 3 or q[2][0] != v[2][0]:
        raise ValueError("q, k must be [B, Hk, Dk] and v [B, Hv, Dv]")
    B, Hk, Dk = q[2]
    Hv, Dv = v[2][1:]
    if len(states[2]) != 4:
        raise ValueError("states must be [pool, Hv, Dk, Dv]")
    _check_contiguous((states[2][0], Hv, Dk, Dv), ("states", states))
    _check_contiguous((B,), ("slots", slots))
    d = _DeltaRuleDesc(_element_type(q[0]), B, 1, Hk, Hv, Dk, Dv, Dk ** -0.5 if scale is None else scale)
    for (name, t), shape in zip(names, ((Hk, Dk), (Hk, Dk), (Hv, Dv), (Hv, Dv))):
        if tuple(t[2]) != (B, *shape):
            raise ValueError(f"{name} must be {[B, *shape]}, not {list(t[2])}")
        setattr(d, name, _strides4(name, (t[0], t[1], (B, 1, *shape), (t[3][0], 0, t[3][1], t[3][2])), (B, 1, *shape)))
    for name, t in (("g", g), ("beta", beta)):
        if t is not None:
            if tuple(t[2]) != (B, Hv):
                raise ValueError(f"{name} must be [B, Hv]")
            setattr(d, name, _Strides(t[3][0], 0, t[3][1]))
    return ctypes.addressof(d), q[1], d


def gated_delta_rule_step(q, k, v, g, beta, states, o, slots=None, scale=None, stream=None):
    """One token of the gated delta rule: q, k [B, Hk, Dk], v, o [B, Hv, Dv], g (or None) and beta float32 [B, Hv]; the states float32
    [pool, Hv, Dk, Dv] of the slots int32 [B] (None: 0 .. B - 1; negative: no sequence) are advanced in place."""
    m = _marshal or _load_marshal()
    tensors = (q, k, v, o, g, beta, states, slots)
    key = ("step", m.key(*tensors), scale := None if scale is None else float(scale))
    plan = _plans.get(key) or _plan(key, _step_plan, tensors, scale)
    st = m.tfno_gated_delta_rule_step(plan[0], q, k, v, g, beta, states, slots, states.size(0), o, _raw_stream(plan[1]) if stream is None else stream)
    if st != OK:
        raise TfnoError(st, "tfno_gated_delta_rule_step")
    return o


def _strides3(name, t, shape):
    """Strides of a [B, T, C] tensor with its last axis contiguous."""
    if tuple(t[2]) != tuple(shape):
        raise ValueError(f"{name} must be {list(shape)}, not {list(t[2])}")
    if shape[2] > 1 and t[3][2] != 1:
        raise ValueError(f"the last axis of {name} must be contiguous")
    return _Strides(t[3][0], t[3][1], 0)


def _recurrence_plan(x, gate, input_gate, rate, y, dx, dgate, dinput_gate, drate, lengths, tape, initial, final, other, normalise):
    names = (("x", x), ("gate", gate), ("input_gate", input_gate), ("y", y), ("dx", dx), ("dgate", dgate), ("dinput_gate", dinput_gate))
    states = (("the initial state", initial), ("the final state or its gradient", final), ("the gradient of the initial state", other))
    _check_types(x, names, f32=(("rate", rate), ("drate", drate)) + states, i32=(("lengths", lengths),), u8=(("the tape", tape),), what="x")
    if len(x[2]) != 3:
        raise ValueError("x must be [B, T, C]")
    B, T, C = x[2]
    d = _RecurrenceDesc(_element_type(x[0], "x"), B, T, C, normalise)
    for name, t in names:
        if t is not None:
            setattr(d, name, _strides3(name, t, (B, T, C)))
    _check_contiguous((C,), ("rate", rate), ("drate", drate))
    _check_contiguous((B, C), *states)
    _check_contiguous((B,), ("lengths", lengths))
    at = ctypes.addressof(d)
    need = _entry("tfno_gated_recurrence_tape_bytes")(at)
    if tape is not None and (len(tape[2]) != 1 or (tape[2][0] > 1 and tape[3][0] != 1) or tape[2][0] < need):
        raise ValueError(f"the tape must be contiguous and hold {need} bytes")
    ask = _entry("tfno_gated_recurrence_workspace_bytes")
    return at, need, ask(at, 0), ask(at, 1), x[1], d


def gated_recurrence_tape(x):
    """A tape for gated_recurrence and gated_recurrence_backward on tensors of the sizes of x [B, T, C]."""
    torch = _torch or _load_torch()
    m = _marshal or _load_marshal()
    key = ("recurrence tape", m.key(x))
    plan = _plans.get(key) or _plan(key, _recurrence_plan, (x, *(None,) * 13), False)
    return torch.empty(plan[1], dtype=torch.uint8, device=x.device)


def gated_recurrence(x, gate, input_gate, rate, y, normalise: bool = False, initial_state=None, final_state=None, lengths=None, tape=None, stream=None):
    """The gated linear recurrence h = exp(l) h + u, y = h, over whole sequences: x, gate, input_gate, y [B, T, C] (float32 or bfloat16, any strides with the last axis
    contiguous).  l = -rate sigmoid(gate) with rate float32 [C], or gate itself where rate is None; u = x, times sigmoid(input_gate) where that is not None, times
    sqrt(1 - exp(2 l)) with `normalise`.  States are float32 [B, C], lengths int32 [B].  With a tape (gated_recurrence_tape) the gradient can be taken afterwards."""
    m = _marshal or _load_marshal()
    tensors = (x, gate, input_gate, rate, y, None, None, None, None, lengths, tape, initial_state, final_state, None)
    key = ("recurrence", m.key(*tensors), normalise := bool(normalise))
    plan = _plans.get(key) or _plan(key, _recurrence_plan, tensors, normalise)
    ensure_workspace(plan[2], x.device)
    st = m.tfno_gated_recurrence(plan[0], x, gate, input_gate, rate, lengths, initial_state, y, final_state, tape, _raw_stream(plan[4]) if stream is None else stream)
    if st != OK:
        raise TfnoError(st, "tfno_gated_recurrence")
    return y


def gated_recurrence_backward(x, gate, input_gate, rate, d_y, dx, dgate, dinput_gate, drate, tape, normalise: bool = False, d_final_state=None,
                              d_initial_state=None, lengths=None, stream=None):
    """Gradients of gated_recurrence with the same inputs, from its tape and the gradients d_y of y and d_final_state of the final state (None: zeros).  drate (float32
    [C], summed over all tokens) and d_initial_state may be None."""
    m = _marshal or _load_marshal()
    tensors = (x, gate, input_gate, rate, d_y, dx, dgate, dinput_gate, drate, lengths, tape, None, d_final_state, d_initial_state)
    key = ("recurrence", m.key(*tensors), normalise := bool(normalise))
    plan = _plans.get(key) or _plan(key, _recurrence_plan, tensors, normalise)
    ensure_workspace(plan[3], x.device)
    st = m.tfno_gated_recurrence_backward(plan[0], x, gate, input_gate, rate, lengths, tape, d_y, d_final_state, dx, dgate, dinput_gate, drate, d_initial_state,
                                          _raw_stream(plan[4]) if stream is None else stream)
    if st != OK:
        raise TfnoError(st, "tfno_gated_recurrence_backward")
    return dx, dgate, dinput_gate, drate


def _recurrence_step_plan(x, gate, input_gate, rate, y, states, slots, normalise):
    names = (("x", x), ("gate", gate), ("input_gate", input_gate), ("y", y))
    _check_types(x, names, f32=(("rate", rate), ("states", states)), i32=(("slots", slots),), what="x")
    if len(x[2]) != 2:
        raise ValueError("x must be [B, C]")
    B, C = x[2]
    if len(states[2]) != 2:
        raise ValueError("states must be [pool, C]")
    d = _RecurrenceDesc(_element_type(x[0], "x"), B, 1, C, normalise)
    for name, t in names:
        if t is not None:
            if len(t[2]) != 2:
                raise ValueError(f"{name} must be {[B, C]}, not {list(t[2])}")
            setattr(d, name, _strides3(name, (t[0], t[1], (t[2][0], 1, t[2][1]), (t[3][0], 0, t[3][1])), (B, 1, C)))
    _check_contiguous((C,), ("rate", rate))
    _check_contiguous((states[2][0], C), ("states", states))
    _check_contiguous((B,), ("slots", slots))
    return ctypes.addressof(d), x[1], d


def gated_recurrence_step(x, gate, input_gate, rate, states, y, normalise: bool = False, slots=None, stream=None):
    """One token of the gated linear recurrence: x, gate, input_gate, y [B, C]; the states float32 [pool, C] of the slots int32 [B] (None: 0 .. B - 1;
    negative: no sequence) are advanced in place."""
    m = _marshal or _load_marshal()
    tensors = (x, gate, input_gate, rate, y, states, slots)
    key = ("recurrence step", m.key(*tensors), normalise := bool(normalise))
    plan = _plans.get(key) or _plan(key, _recurrence_step_plan, tensors, normalise)
    st = m.tfno_gated_recurrence_step(plan[0], x, gate, input_gate, rate, states, slots, states.size(0), y, _raw_stream(plan[1]) if stream is None else stream)
    if st != OK:
        raise TfnoError(st, "tfno_gated_recurrence_step")
    return y


# ---------------------------------------------------------------- between two blocks

_ACTIVATIONS = {"none": 0, "silu": 1, "sigmoid": 2}


def _block_norm_ways(norm_after, activation, residual_scale, eps):
    if activation not in _ACTIVATIONS:
        raise ValueError(f"activation must be one of {list(_ACTIVATIONS)}")
    return bool(norm_after), _ACTIVATIONS[activation], float(residual_scale), float(eps)


def _block_norm_plan(y, r, gate, w_after, w_before, r_out, n_out, dy, dr, dgate, dw_after, dw_before, lengths, norm_after, activation, residual_scale, eps):
    torch = _torch or _load_torch()
    if len(y[2]) != 3:
        raise ValueError("y must be [B, T, C]")
    B, T, C = y[2]
    kind = 0 if gate is None else {3: 1, 2: 2, 1: 3}.get(len(gate[2]), -1)
    if kind < 0:
        raise ValueError("gate must be [B, T, C], [B, C] or [C]")
    gates, weights = (("gate", gate), ("dgate", dgate)), (("w_after", w_after), ("w_before", w_before), ("dw_after", dw_after), ("dw_before", dw_before))
    _check_types(y, (("y", y), ("n_out", n_out), ("dy", dy)) + (gates if kind == 1 else ()), f32=weights + (gates if kind != 1 else ()),
                 i32=(("lengths", lengths),), what="y")
    residuals = (("r", r), ("r_out", r_out), ("dr", dr))
    residual = next((t for _, t in residuals if t is not None), y)
    if residual[0] is not y[0] and residual[0] is not torch.float32:
        raise TypeError(f"r must be {y[0]} or float32")
    _check_types(residual, residuals, what="y")
    if residual[1] != y[1]:
        raise TypeError("r and r_out must be tensors on the device of y")
    d = _BlockNormDesc(_element_type(y[0], "y"), _element_type(residual[0], "r"), B, T, C, kind, activation, norm_after, residual_scale, eps)
    for name, t in (("y", y), ("n_out", n_out), ("dy", dy)) + residuals + (gates if kind == 1 else ()):
        if t is not None:
            setattr(d, name, _strides3(name, t, (B, T, C)))
    if kind == 2:
        if tuple(gate[2]) != (B, C) or (C > 1 and gate[3][1] != 1):
            raise ValueError("the gate of sequences must be [B, C] with contiguous rows")
        d.gate = _Strides(gate[3][0], 0, 0)
        _check_contiguous((B, C), ("dgate", dgate))
        d.dgate = _Strides(C, 0, 0)
    elif kind != 1:
        _check_contiguous((C,), *gates)
    _check_contiguous((C,), *weights)
    _check_contiguous((B,), ("lengths", lengths))
    at = ctypes.addressof(d)
    sums = dw_after is not None or dw_before is not None or (dgate is not None and kind != 1)
    return at, _entry("tfno_block_norm_workspace_bytes")(at) if sums else 0, y[1], d


def block_norm(y, r, gate, w_after, w_before, r_out, n_out, norm_after: bool = True, activation="none", residual_scale: float = 1.0, eps: float = 1e-6,
               lengths=None, stream=None):
    """What stands between two blocks, in one pass: r_out = residual_scale r + act(gate) Norm(y) w_after and n_out = Norm(r_out) w_before, where
    Norm(x) = x / sqrt(mean x^2 + eps).  y, n_out [B, T, C] float32 or bfloat16, r and r_out of that type or float32, any strides with the last axis contiguous; gate [B, T, C]
    of y's type, or float32 [B, C] or [C], or None; activation "none", "silu" or "sigmoid"; weights float32 [C] or None (ones).  Without norm_after y goes in as it
    is; r, and either result, may be None.  r_out may be r and n_out y."""
    m = _marshal or _load_marshal()
    tensors = (y, r, gate, w_after, w_before, r_out, n_out, None, None, None, None, None, lengths)
    ways = _block_norm_ways(norm_after, activation, residual_scale, eps)
    key = ("block norm", m.key(*tensors), ways)
    plan = _plans.get(key) or _plan(key, _block_norm_plan, tensors, *ways)
    st = m.tfno_block_norm(plan[0], y, r, gate, w_after, w_before, lengths, r_out, n_out, _raw_stream(plan[2]) if stream is None else stream)
    if st != OK:
        raise TfnoError(st, "tfno_block_norm")
    return r_out, n_out


def block_norm_backward(y, r, gate, w_after, w_before, d_r_out, d_n_out, dy, dr, dgate, dw_after, dw_before, norm_after: bool = True, activation="none",
                        residual_scale: float = 1.0, eps: float = 1e-6, lengths=None, stream=None):
    """Gradients of block_norm with the same inputs from those of its results, d_r_out and d_n_out (None: zeros).  dr, dgate, dw_after and dw_before may be None; a
    gradient of weights or of a gate that tokens share is float32 and summed over them.  dr may be d_r_out and dy d_n_out."""
    m = _marshal or _load_marshal()
    tensors = (y, r, gate, w_after, w_before, d_r_out, d_n_out, dy, dr, dgate, dw_after, dw_before, lengths)
    ways = _block_norm_ways(norm_after, activation, residual_scale, eps)
    key = ("block norm", m.key(*tensors), ways)
    plan = _plans.get(key) or _plan(key, _block_norm_plan, tensors, *ways)
    ensure_workspace(plan[1], y.device)
    st = m.tfno_block_norm_backward(plan[0], y, r, gate, w_after, w_before, lengths, d_r_out, d_n_out, dy, dr, dgate, dw_after, dw_before,
                                    _raw_stream(plan[2]) if stream is None else stream)
    if st != OK:
        raise TfnoError(st, "tfno_block_norm_backward")
    return dy, dr, dgate, dw_after, dw_before


# ---------------------------------------------------------------- gradients

def clip_grad_norm(gradients, limit: float, norm=None, stream=None):
    """Scales the gradients (float32, bfloat16 or complex64 tensors on one device, each filling its own memory) in place so that the norm over all their elements is at
    most `limit`; math.inf gives the norm alone.  A gradient may be None (of a parameter that has none).  norm: one float32 on the device for the norm before that, or None.
    Gradients whose norm is not finite stay as they are."""
    m = _marshal or _load_marshal()
    gradients = gradients if isinstance(gradients, (list, tuple)) else list(gradients)
    first = norm if norm is not None else next((g for g in gradients if g is not None), None)
    if first is None:
        return norm
    device = first.device
    if device.type != "cuda":
        raise TypeError("gradients must be tensors on the device")
    ensure_workspace(_entry("tfno_clip_grad_norm_workspace_bytes")(len(gradients)), device)
    st = m.tfno_clip_grad_norm(gradients, limit, norm, device.index, _raw_stream(device.index) if stream is None else stream)
    if st != OK:
        raise TfnoError(st, "tfno_clip_grad_norm")
    return norm
