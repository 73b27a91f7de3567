"""ctypes binding of libab.so: same names as the C entry points (include/ab.h), argument
marshalling only.  Tensors are torch CUDA tensors (torch supplies device memory and streams);
every step of the computation runs in the library's kernels.  There is no CPU path: loading
fails loudly when the library has not been built, and every call raises on a negative status.
"""
from __future__ import annotations

import ctypes
import os
from ctypes import c_char_p, c_float, c_int, c_int64, c_size_t, c_void_p

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libab.so")

AB_F32, AB_BF16 = 0, 1
AB_OP_LAYER_FORWARD, AB_OP_LAYER_BACKWARD, AB_OP_GROUP_AVERAGE, AB_OP_RECOMBINE, AB_OP_SVD_SPLIT = range(5)
AB_OP_DENSE_FORWARD, AB_OP_DENSE_BACKWARD = 5, 6
AB_OK = 0
AB_ERR_INVALID_ARG, AB_ERR_UNSUPPORTED, AB_ERR_WORKSPACE = -1, -2, -3
AB_ERR_NOT_CONVERGED, AB_ERR_TIMEOUT, AB_ERR_CUDA, AB_ERR_ACCURACY = -4, -5, -6, -7
AB_SYNC_AUTO, AB_SYNC_DENSE, AB_SYNC_FACTORED = 0, 1, 2

EXPORTS = ["ab_status_string", "ab_version", "ab_launch_count", "ab_workspace_bytes", "ab_layer_forward", "ab_layer_backward",
           "ab_group_average", "ab_recombine", "ab_svd_split", "ab_group_sync", "ab_sync_workspace_bytes",
           "ab_layer_forward_static", "ab_static_scratch_elems", "ab_adamw_step", "ab_lr_rebound_factor", "ab_selftest_bounded_wait",
           "ab_selftest_chain_stall", "ab_selftest_chain_stall_workspace_bytes",
           "ab_selftest_split_fallback", "ab_selftest_split_fallback_workspace_bytes",
           "ab_dense_forward", "ab_dense_backward", "ab_conv3x3_forward", "ab_conv3x3_backward",
           "ab_conv3x3_workspace_bytes", "ab_recombine_mean", "ab_adapter_forward", "ab_adapter_backward",
           "ab_adapter_workspace_bytes", "ab_selftest_adapter_form", "ab_grad_clip", "ab_grad_clip_workspace_bytes"]


class AbError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} ({status})")


class ab_sync_desc(ctypes.Structure):
    _fields_ = [("A_copies", c_void_p), ("B_copies", c_void_p), ("strideA", c_int64), ("strideB", c_int64),
                ("m", c_int), ("n", c_int), ("r", c_int), ("A_out", c_void_p), ("B_out", c_void_p),
                ("sigma", c_void_p), ("r_out", c_void_p), ("W_out", c_void_p)]


class ab_clip_desc(ctypes.Structure):
    _fields_ = [("grad", c_void_p), ("out", c_void_p), ("count", c_int64)]


_lib = None


def lib() -> ctypes.CDLL:
    """The loaded library.  Raises if it has not been built (python -m paper_2405_01067_b200.build)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python paper_2405_01067_b200/build.py`; "
                           "there is no fallback path")
    L = ctypes.CDLL(LIB_PATH)
    L.ab_status_string.restype = c_char_p
    L.ab_status_string.argtypes = [c_int]
    L.ab_version.restype = c_char_p
    L.ab_launch_count.restype = ctypes.c_longlong
    L.ab_workspace_bytes.restype = c_size_t
    L.ab_workspace_bytes.argtypes = [c_int, c_int64, c_int, c_int, c_int, c_int, c_int]
    L.ab_layer_forward.restype = c_int
    L.ab_layer_forward.argtypes = [c_void_p] * 5 + [c_int64] + [c_int] * 6 + [c_void_p, c_size_t, c_void_p]
    L.ab_layer_backward.restype = c_int
    L.ab_layer_backward.argtypes = [c_void_p] * 8 + [c_int64] + [c_int] * 6 + [c_void_p, c_size_t, c_void_p]
    L.ab_adapter_forward.restype = c_int
    L.ab_adapter_forward.argtypes = [c_void_p] * 8 + [c_int64] + [c_int] * 4 + [c_int64] * 2 + [c_int, c_void_p, c_size_t, c_void_p]
    L.ab_adapter_backward.restype = c_int
    L.ab_adapter_backward.argtypes = [c_void_p] * 11 + [c_int64] + [c_int] * 4 + [c_int64] * 2 + [c_int, c_void_p, c_size_t, c_void_p]
    L.ab_selftest_adapter_form.restype = c_int
    L.ab_selftest_adapter_form.argtypes = [c_int64, c_int, c_int]
    L.ab_adapter_workspace_bytes.restype = c_size_t
    L.ab_adapter_workspace_bytes.argtypes = [c_int64] + [c_int] * 5
    L.ab_group_average.restype = c_int
    L.ab_group_average.argtypes = [c_void_p, c_int64, c_int, c_int64, c_int, c_int, c_void_p, c_void_p]
    L.ab_recombine.restype = c_int
    L.ab_recombine.argtypes = [c_void_p, c_void_p, c_void_p] + [c_int] * 6 + [c_void_p, c_size_t, c_void_p]
    L.ab_svd_split.restype = c_int
    L.ab_svd_split.argtypes = [c_void_p, c_int, c_int, c_int, c_float] + [c_void_p] * 5 + [c_int, c_int,
                                                                                         c_void_p, c_size_t, c_void_p]
    L.ab_group_sync.restype = c_int
    L.ab_group_sync.argtypes = [ctypes.POINTER(ab_sync_desc), c_int, c_int, c_float, c_int, c_void_p, c_void_p,
                                c_size_t, c_void_p, c_int]
    L.ab_sync_workspace_bytes.restype = c_size_t
    L.ab_sync_workspace_bytes.argtypes = [ctypes.POINTER(ab_sync_desc), c_int, c_int, c_int]
    L.ab_layer_forward_static.restype = c_int
    L.ab_layer_forward_static.argtypes = [c_void_p] * 4 + [c_int64] + [c_int] * 6 + [c_void_p]
    L.ab_static_scratch_elems.restype = c_size_t
    L.ab_adamw_step.restype = c_int
    L.ab_adamw_step.argtypes = [c_void_p] * 5 + [c_int64] + [c_float] * 5 + [c_int, c_void_p]
    L.ab_grad_clip.restype = c_int
    L.ab_grad_clip.argtypes = [ctypes.POINTER(ab_clip_desc), c_int, c_float, c_void_p, c_int, c_void_p, c_size_t, c_void_p]
    L.ab_grad_clip_workspace_bytes.restype = c_size_t
    L.ab_grad_clip_workspace_bytes.argtypes = [c_int]
    L.ab_lr_rebound_factor.restype = c_float
    L.ab_lr_rebound_factor.argtypes = [c_int, c_int, c_float]
    L.ab_selftest_bounded_wait.restype = c_int
    L.ab_selftest_bounded_wait.argtypes = [c_void_p, ctypes.c_uint, c_void_p]
    L.ab_selftest_chain_stall.restype = c_int
    L.ab_selftest_chain_stall.argtypes = [c_void_p, c_size_t, ctypes.c_uint, c_void_p]
    L.ab_selftest_chain_stall_workspace_bytes.restype = c_size_t
    L.ab_selftest_split_fallback.restype = c_int
    L.ab_selftest_split_fallback.argtypes = [c_void_p] + [c_int] * 4 + [ctypes.c_ulonglong, c_int] + [c_void_p] * 6 + [c_size_t, c_void_p]
    L.ab_selftest_split_fallback_workspace_bytes.restype = c_size_t
    L.ab_selftest_split_fallback_workspace_bytes.argtypes = [c_int] * 4
    L.ab_dense_forward.restype = c_int
    L.ab_dense_forward.argtypes = [c_void_p] * 3 + [c_int64, c_int, c_int, c_int, c_void_p, c_size_t, c_void_p]
    L.ab_dense_backward.restype = c_int
    L.ab_dense_backward.argtypes = [c_void_p] * 5 + [c_int64, c_int, c_int, c_int, c_void_p, c_size_t, c_void_p]
    L.ab_conv3x3_forward.restype = c_int
    L.ab_conv3x3_forward.argtypes = [c_void_p] * 5 + [c_int] * 9 + [c_void_p, c_size_t, c_void_p]
    L.ab_conv3x3_backward.restype = c_int
    L.ab_conv3x3_backward.argtypes = [c_void_p] * 8 + [c_int] * 9 + [c_void_p, c_size_t, c_void_p]
    L.ab_conv3x3_workspace_bytes.restype = c_size_t
    L.ab_conv3x3_workspace_bytes.argtypes = [c_int] * 6
    L.ab_recombine_mean.restype = c_int
    L.ab_recombine_mean.argtypes = [c_void_p, c_int64, c_void_p, c_int64, c_int, c_void_p, c_void_p, c_void_p,
                                    c_int, c_int, c_int, c_int, c_void_p]
    _lib = L
    return L


def ab_selftest_bounded_wait(limit_us: int = 1000, stream=None) -> int:
    """Runs the bounded-wait self-test and returns the device status it left (AB_ERR_TIMEOUT when the wait
    gave up as designed).  Synchronises."""
    status = torch.zeros((1,), dtype=torch.int32, device="cuda")
    _check(lib().ab_selftest_bounded_wait(_ptr(status), int(limit_us), _stream(stream)), "ab_selftest_bounded_wait")
    return int(status.item())


def ab_selftest_chain_stall(limit_us: int = 1000, stream=None) -> int:
    """Runs the fused chain kernel with its loader switched off and returns the device status its unwinding
    left (AB_ERR_TIMEOUT).  Synchronises."""
    ws = workspace(int(lib().ab_selftest_chain_stall_workspace_bytes()), "cuda")
    _check(lib().ab_selftest_chain_stall(_ptr(ws), ws.numel(), int(limit_us), _stream(stream)), "ab_selftest_chain_stall")
    return workspace_status(ws)


def ab_selftest_split_fallback(W, r_max: int, flagged: int, solver_status: int = AB_OK, stream=None):
    """Splits W (count, m, n) with the matrices of `flagged` (a bit each) sent through the Jacobi fallback.  Returns (A, B,
    sigma, r_out, status), a matrix per row."""
    _dev_ok(W)
    count, m, n = W.shape
    dev = W.device
    A, B = torch.empty((count, m, r_max), device=dev), torch.empty((count, r_max, n), device=dev)
    sigma = torch.empty((count, min(r_max, m, n)), device=dev)
    r_out, status = (torch.zeros((count,), dtype=torch.int32, device=dev) for _ in range(2))
    ws = workspace(int(lib().ab_selftest_split_fallback_workspace_bytes(m, n, r_max, count)), dev)
    _check(lib().ab_selftest_split_fallback(_ptr(W), m, n, r_max, count, int(flagged), int(solver_status), _ptr(A), _ptr(B), _ptr(sigma),
                                            _ptr(r_out), _ptr(status), _ptr(ws), ws.numel(), _stream(stream)),
           "ab_selftest_split_fallback")
    return A, B, sigma, r_out, status


def ab_launch_count() -> int:
    return int(lib().ab_launch_count())


def status_string(status: int) -> str:
    return lib().ab_status_string(int(status)).decode()


def _dt(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return AB_F32
    if t.dtype == torch.bfloat16:
        return AB_BF16
    raise TypeError(f"unsupported dtype {t.dtype}")


# Addresses and streams go to ctypes as plain integers, which it converts itself, and the current stream is asked for by its
# handle: a Stream object costs 3 us and a c_void_p per argument 2 us more, of a call that took 15 us on the host.
def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream(stream):
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device()) if stream is None else stream.cuda_stream


def _check(status: int, where: str):
    if status != AB_OK:
        raise AbError(status, where)


def _dev_ok(*ts):
    for t in ts:
        if t is not None and (not t.is_cuda or not t.is_contiguous()):
            raise ValueError("tensors must be contiguous CUDA tensors")


def workspace(nbytes: int, device) -> torch.Tensor:
    """A 256-byte aligned scratch buffer of at least nbytes (torch's allocator aligns to 512)."""
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


# What a call makes itself on a stream of the caller's is taken from that stream's own memory: a block of the current stream's could
# still be in use there, by work that the caller's stream does not wait for, and would go back to the current stream as soon as its tensor
# is dropped, while the call is still to run.
def _scratch(nbytes, device, stream):
    """A workspace that a call owns."""
    if stream is None:
        return workspace(nbytes, device)
    with torch.cuda.stream(stream):
        return workspace(nbytes, device)


def _result(x, shape, stream, dtype=None, zero=False):
    """A tensor on x's device (of x's type, unless given) that a call returns: the caller reads it on the current stream, behind a wait
    of theirs, and its memory is kept until that has run too."""
    if stream is None:
        return x.new_zeros(shape, dtype=dtype) if zero else x.new_empty(shape, dtype=dtype)
    here = torch.cuda.current_stream(x.device)
    with torch.cuda.stream(stream):
        t = x.new_zeros(shape, dtype=dtype) if zero else x.new_empty(shape, dtype=dtype)
    t.record_stream(here)
    return t


def workspace_status(ws: torch.Tensor) -> int:
    """Device status word a layer call left at the head of its workspace (synchronises)."""
    return int(ws[:4].view(torch.int32).item())


def ab_workspace_bytes(op: int, N: int, m: int, n: int, r: int, K: int = 1, dt: int = AB_F32) -> int:
    return int(lib().ab_workspace_bytes(op, N, m, n, r, K, dt))


def ab_layer_forward(x, A, B, y=None, T_save=None, ws=None, stream=None, save_T=False):
    """y = (x B^T) A^T.  Returns (y, T_save or None)."""
    _dev_ok(x, A, B, y, T_save)
    N, n = x.shape
    m, r = A.shape
    dt = _dt(x)
    if y is None:
        y = _result(x, (N, m), stream)
    if save_T and T_save is None:
        T_save = _result(x, (N, r), stream)
    if ws is None:
        ws = _scratch(ab_workspace_bytes(AB_OP_LAYER_FORWARD, N, m, n, r, 1, dt), x.device, stream)
    st = lib().ab_layer_forward(_ptr(x), _ptr(A), _ptr(B), _ptr(y), _ptr(T_save), N, m, n, r,
                                A.stride(0), B.stride(0), dt, _ptr(ws), ws.numel(), _stream(stream))
    _check(st, "ab_layer_forward")
    return y, T_save


def ab_layer_forward_static(x, A, B, y, stream=None):
    """y = (x B^T) A^T with the intermediate in the library's built-in scratch array: for callers that
    cannot allocate a workspace.  `y` must be supplied (this call allocates nothing); N*r is limited to
    ab_static_scratch_elems().  Calls that may overlap on the GPU race on the shared array."""
    _dev_ok(x, A, B, y)
    N, n = x.shape
    m, r = A.shape
    st = lib().ab_layer_forward_static(_ptr(x), _ptr(A), _ptr(B), _ptr(y), N, m, n, r, A.stride(0), B.stride(0),
                                       _dt(x), _stream(stream))
    _check(st, "ab_layer_forward_static")
    return y


def ab_layer_backward(x, dY, A, B, T_saved=None, want=("dX", "dA", "dB"), dX=None, dA=None, dB=None,
                      ws=None, stream=None):
    """dX = (dY A) B, dA = dY^T T, dB = (dY A)^T x.  Returns (dX, dA, dB); entries not in `want` are None."""
    _dev_ok(x, dY, A, B, T_saved, dX, dA, dB)
    N, n = x.shape
    m, r = A.shape
    dt = _dt(x)
    if "dX" in want and dX is None:
        dX = _result(x, (N, n), stream)
    if "dA" in want and dA is None:
        dA = _result(x, (m, r), stream, torch.float32)
    if "dB" in want and dB is None:
        dB = _result(x, (r, n), stream, torch.float32)
    if ws is None:
        ws = _scratch(ab_workspace_bytes(AB_OP_LAYER_BACKWARD, N, m, n, r, 1, dt), x.device, stream)
    st = lib().ab_layer_backward(_ptr(x), _ptr(dY), _ptr(A), _ptr(B), _ptr(T_saved), _ptr(dX), _ptr(dA), _ptr(dB),
                                 N, m, n, r, A.stride(0), B.stride(0), dt, _ptr(ws), ws.numel(), _stream(stream))
    _check(st, "ab_layer_backward")
    return dX, dA, dB


def ab_conv3x3_workspace_bytes(batch, H, W, C, m, r) -> int:
    return int(lib().ab_conv3x3_workspace_bytes(batch, H, W, C, m, r))


def ab_conv3x3_forward(x, A, B, y=None, T_save=None, ws=None, stream=None, save_T=False):
    """Factorised 3 x 3 convolution on an NHWC activation x [batch, H, W, C].  Returns (y [batch,H,W,m], T or None)."""
    _dev_ok(x, A, B, y, T_save)
    batch, H, W, C = x.shape
    m, r = A.shape
    if y is None:
        y = _result(x, (batch, H, W, m), stream)
    if save_T and T_save is None:
        T_save = _result(x, (batch * H * W, r), stream)
    if ws is None:
        ws = _scratch(ab_conv3x3_workspace_bytes(batch, H, W, C, m, r), x.device, stream)
    st = lib().ab_conv3x3_forward(_ptr(x), _ptr(A), _ptr(B), _ptr(y), _ptr(T_save), batch, H, W, C, m, r,
                                  A.stride(0), B.stride(0), _dt(x), _ptr(ws), ws.numel(), _stream(stream))
    _check(st, "ab_conv3x3_forward")
    return y, T_save


def ab_conv3x3_backward(x, dY, A, B, T_saved=None, want=("dX", "dA", "dB"), dX=None, dA=None, dB=None, ws=None,
                        stream=None):
    """dX [batch,H,W,C], dA [m,r], dB [r,9C] of the factorised convolution; dY is [batch,H,W,m]."""
    _dev_ok(x, dY, A, B, T_saved, dX, dA, dB)
    batch, H, W, C = x.shape
    m, r = A.shape
    if "dX" in want and dX is None:
        dX = _result(x, x.shape, stream)
    if "dA" in want and dA is None:
        dA = _result(x, (m, r), stream, torch.float32)
    if "dB" in want and dB is None:
        dB = _result(x, (r, 9 * C), stream, torch.float32)
    if ws is None:
        ws = _scratch(ab_conv3x3_workspace_bytes(batch, H, W, C, m, r), x.device, stream)
    st = lib().ab_conv3x3_backward(_ptr(x), _ptr(dY), _ptr(A), _ptr(B), _ptr(T_saved), _ptr(dX), _ptr(dA), _ptr(dB),
                                   batch, H, W, C, m, r, A.stride(0), B.stride(0), _dt(x), _ptr(ws), ws.numel(),
                                   _stream(stream))
    _check(st, "ab_conv3x3_backward")
    return dX, dA, dB


def ab_dense_forward(x, W, y=None, ws=None, stream=None):
    """y = x W^T with W held dense (the full-rank phases of a cycle)."""
    _dev_ok(x, W, y)
    N, n = x.shape
    m = W.shape[0]
    dt = _dt(x)
    if y is None:
        y = _result(x, (N, m), stream)
    if ws is None:
        ws = _scratch(ab_workspace_bytes(AB_OP_DENSE_FORWARD, N, m, n, 0, 1, dt), x.device, stream)
    st = lib().ab_dense_forward(_ptr(x), _ptr(W), _ptr(y), N, m, n, dt, _ptr(ws), ws.numel(), _stream(stream))
    _check(st, "ab_dense_forward")
    return y


def ab_dense_backward(x, dY, W, want=("dX", "dW"), dX=None, dW=None, ws=None, stream=None):
    """dX = dY W, dW = dY^T x (fp32).  Returns (dX, dW); entries not in `want` are None."""
    _dev_ok(x, dY, W, dX, dW)
    N, n = x.shape
    m = W.shape[0]
    dt = _dt(x)
    if "dX" in want and dX is None:
        dX = _result(x, (N, n), stream)
    if "dW" in want and dW is None:
        dW = _result(x, (m, n), stream, torch.float32)
    if ws is None:
        ws = _scratch(ab_workspace_bytes(AB_OP_DENSE_BACKWARD, N, m, n, 0, 1, dt), x.device, stream)
    st = lib().ab_dense_backward(_ptr(x), _ptr(dY), _ptr(W), _ptr(dX), _ptr(dW), N, m, n, dt, _ptr(ws), ws.numel(),
                                 _stream(stream))
    _check(st, "ab_dense_backward")
    return dX, dW


def ab_adapter_workspace_bytes(x, A, B) -> int:
    """Scratch bytes of ab_adapter_forward and ab_adapter_backward for rows x (N, n) and adapters A (L, m, r), B (L, r, n)."""
    L, m, r = A.shape
    return int(lib().ab_adapter_workspace_bytes(x.shape[0], m, B.shape[2], r, L, _dt(x)))


# What the adapter calls look at in every tensor, in the order of what is cheap: a serving step is a call of 10 us on the device.
# get_device() is -1 for a tensor that is not on a GPU.
def _fits(what, t, shape, dtype, dev):
    if t.shape != shape or t.dtype != dtype or not t.is_contiguous() or t.get_device() != dev:
        raise ValueError(f"{what}: expected a contiguous {dtype} tensor of {tuple(shape)} on the current device (cuda:{dev}), "
                         f"got {t.dtype} {tuple(t.shape)} on {t.device}, strides {t.stride()}")


def _adapter_ws(ws, x, A, B, dev, stream):
    """The workspace of an adapter call: the caller's, or one of the call's own."""
    if ws is None:
        return _scratch(ab_adapter_workspace_bytes(x, A, B), x.device, stream)
    if ws.get_device() != dev or not ws.is_contiguous():
        raise ValueError(f"ws: expected a contiguous tensor on the current device (cuda:{dev}), got one on {ws.device}, strides {ws.stride()}")
    return ws


def _adapter_ok(x, W, A, B, row_adapter, scale):
    """Checks the inputs of an adapter call; returns (N, n, L, m, r, device).  A and B may be spaced along their first axis."""
    if x.dim() != 2 or A.dim() != 3:
        raise ValueError("x is (N, n), A (L, m, r)")
    N, n = x.shape
    L, m, r = A.shape
    dt, dev = x.dtype, torch._C._cuda_getDevice()
    _fits("x", x, (N, n), dt, dev)
    if W is not None:
        _fits("W", W, (m, n), dt, dev)
    _fits("row_adapter", row_adapter, (N,), torch.int32, dev)
    if scale is not None:
        _fits("scale", scale, (L,), torch.float32, dev)
    if B.shape != (L, r, n):
        raise ValueError(f"B {tuple(B.shape)} does not fit A {tuple(A.shape)} and rows of {n}")
    for t, cols in ((A, r), (B, n)):
        _, s1, s2 = t.stride()
        if t.dtype != dt or t.get_device() != dev or s1 != cols or s2 != 1:
            if not (t.dtype == dt and t.get_device() == dev and (L == 0 or t[0].is_contiguous())):
                raise ValueError("A and B have x's type and device, and each adapter's matrix is contiguous")
    return N, n, L, m, r, dev


def ab_adapter_forward(x, W, A, B, row_adapter, scale=None, y=None, T_save=None, ws=None, stream=None, save_T=False):
    """y_i = W x_i + scale_a A_a (B_a x_i) with a = row_adapter[i] (-1: W x_i alone).  x (N, n), W (m, n), A (L, m, r),
    B (L, r, n), row_adapter int32 (N,), scale fp32 (L,) or None.  Returns (y, T (N, r) fp32 or None)."""
    if W is None:
        raise ValueError("the shared projection W is wanted in a forward call")
    N, n, L, m, r, dev = _adapter_ok(x, W, A, B, row_adapter, scale)
    if y is None:
        y = x.new_empty((N, m)) if stream is None else _result(x, (N, m), stream)
    else:
        _fits("y", y, (N, m), x.dtype, dev)
    if T_save is not None:
        _fits("T_save", T_save, (N, r), torch.float32, dev)
    elif save_T:
        T_save = _result(x, (N, r), stream, torch.float32)
    ws = _adapter_ws(ws, x, A, B, dev, stream)
    st = lib().ab_adapter_forward(x.data_ptr(), W.data_ptr(), A.data_ptr(), B.data_ptr(), _ptr(scale), row_adapter.data_ptr(), y.data_ptr(),
                                  _ptr(T_save), N, m, n, r, L, A.stride(0), B.stride(0), _dt(x), ws.data_ptr(), ws.numel(),
                                  torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream.cuda_stream)
    if st != AB_OK:
        raise AbError(st, "ab_adapter_forward")
    return y, T_save


def ab_adapter_backward(x, dY, W, A, B, row_adapter, scale=None, T_saved=None, want=("dX", "dA", "dB"), dX=None, dA=None, dB=None,
                        ws=None, stream=None):
    """Gradients of ab_adapter_forward: dX (N, n), dA (L, m, r) and dB (L, r, n) in fp32; entries not in `want` are None.  T_saved is
    the T of the forward call, or None to recompute it.  W may be None where dX is not wanted."""
    N, n, L, m, r, dev = _adapter_ok(x, W, A, B, row_adapter, scale)
    _fits("dY", dY, (N, m), x.dtype, dev)
    if T_saved is not None:
        _fits("T_saved", T_saved, (N, r), torch.float32, dev)
    if dX is not None:
        _fits("dX", dX, (N, n), x.dtype, dev)
    elif "dX" in want:
        dX = x.new_empty((N, n)) if stream is None else _result(x, (N, n), stream)
    if dA is not None:
        _fits("dA", dA, (L, m, r), torch.float32, dev)
    elif "dA" in want:
        dA = _result(x, (L, m, r), stream, torch.float32)
    if dB is not None:
        _fits("dB", dB, (L, r, n), torch.float32, dev)
    elif "dB" in want:
        dB = _result(x, (L, r, n), stream, torch.float32)
    ws = _adapter_ws(ws, x, A, B, dev, stream)
    st = lib().ab_adapter_backward(x.data_ptr(), dY.data_ptr(), _ptr(W), A.data_ptr(), B.data_ptr(), _ptr(scale), row_adapter.data_ptr(),
                                   _ptr(T_saved), _ptr(dX), _ptr(dA), _ptr(dB), N, m, n, r, L, A.stride(0), B.stride(0), _dt(x),
                                   ws.data_ptr(), ws.numel(),
                                   torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream.cuda_stream)
    if st != AB_OK:
        raise AbError(st, "ab_adapter_backward")
    return dX, dA, dB


def ab_adamw_step(param, grad, m, v, lr, step, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=1e-2, param_bf16=None,
                  stream=None):
    """One AdamW update in place (param, m, v fp32; grad fp32); param_bf16 optionally receives the rounded copy."""
    _dev_ok(param, grad, m, v, param_bf16)
    for t in (param, grad, m, v):
        if t.dtype != torch.float32 or not t.is_contiguous():
            raise ValueError("ab_adamw_step takes contiguous fp32 tensors")
    if param_bf16 is not None and (param_bf16.dtype != torch.bfloat16 or param_bf16.numel() != param.numel()):
        raise ValueError("param_bf16 must be a bf16 tensor of the same size")
    st = lib().ab_adamw_step(_ptr(param), _ptr(grad), _ptr(m), _ptr(v), _ptr(param_bf16), param.numel(), lr, beta1, beta2,
                             eps, weight_decay, step, _stream(stream))
    _check(st, "ab_adamw_step")
    return param


class ClipPlan:
    """Descriptors of the clipping of one step's gradients (ab_grad_clip): tensors of one type at addresses that stay, as an optimizer's do.
    Gradients that are made anew every step (set to None behind it) go to ab_grad_clip themselves: a plan kept over them scales the old ones.  out:
    tensors that receive the scaled values (None: in place); norm_only leaves the gradients alone.  norm: what the last call returned."""

    def __init__(self, grads, out=None, norm_only=False):
        self.grads = list(grads)
        self.out = None if norm_only else self.grads if out is None else list(out)
        if not self.grads:
            raise ValueError("no gradients")
        outs = self.out if self.out is not None else [None] * len(self.grads)
        if len(outs) != len(self.grads):
            raise ValueError("as many outputs as gradients")
        dev = torch.cuda.current_device()
        self.dt = _dt(self.grads[0])
        for g, o in zip(self.grads, outs):
            _dev_ok(g, o)
            if g.dtype != self.grads[0].dtype or (o is not None and (o.dtype != g.dtype or o.numel() != g.numel())):
                raise ValueError("gradients and outputs have one type, and each output its gradient's size")
            if g.device.index != dev or (o is not None and o.device.index != dev):
                raise ValueError("tensors must be on the current device")
        self.descs = (ab_clip_desc * len(self.grads))(*[(g.data_ptr(), None if o is None else o.data_ptr(), g.numel())
                                                        for g, o in zip(self.grads, outs)])
        self.dev, self.count, self.ws_bytes = dev, len(self.grads), lib().ab_grad_clip_workspace_bytes(len(self.grads))
        # Of calls on the stream that the plan was made on: they come one after the other, in one workspace.  Norms, each for one call, are cut
        # 64 at a time (an allocation a call takes 2.5 us of 9).
        self.stream, self.ws, self.norms = torch._C._cuda_getCurrentRawStream(dev), None, []
        self.norm = None

    def _more(self):
        if self.ws is None:
            self.ws = workspace(self.ws_bytes, self.grads[0].device)
        self.norms = list(torch.empty(64, dtype=torch.float32, device=self.grads[0].device).unbind())


def ab_grad_clip(plan, max_norm: float, stream=None):
    """Scales the gradients of a ClipPlan, or those of a list in place, by max_norm / norm where their global norm is above max_norm.  Returns
    (outputs or None, norm), norm a device tensor of one fp32 value, of this call alone; one that is not finite scales nothing.  The plan
    may go when the call returns; its tensors stay until the stream has run it."""
    if not isinstance(plan, ClipPlan):
        plan = ClipPlan(plan)
    dev = torch._C._cuda_getDevice()
    if plan.dev != dev:
        raise ValueError("the plan's tensors must be on the current device")
    raw = torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream.cuda_stream
    if stream is None and raw == plan.stream and not torch._C._cuda_isCurrentStreamCapturing():
        if not plan.norms:
            plan._more()
        norm, ws = plan.norms.pop(), plan.ws
    else:   # another stream, or a captured call, which may be replayed on any
        norm, ws = _result(plan.grads[0], (), stream, torch.float32), _scratch(plan.ws_bytes, plan.grads[0].device, stream)
    st = lib().ab_grad_clip(plan.descs, plan.count, float(max_norm), norm.data_ptr(), plan.dt, ws.data_ptr(), plan.ws_bytes, raw)
    if st != AB_OK:
        raise AbError(st, "ab_grad_clip")
    plan.norm = norm
    return plan.out, norm


def ab_lr_rebound_factor(steps_since_change: int, rebound_steps: int, floor: float = 0.0) -> float:
    return float(lib().ab_lr_rebound_factor(steps_since_change, rebound_steps, floor))


def ab_group_average(copies, out=None, out_dtype=None, stream=None):
    """Mean over the leading axis of a (K, ...) tensor, fp32 sum in ascending k."""
    _dev_ok(copies, out)
    K = copies.shape[0]
    count = copies[0].numel()
    if out is None:
        out = _result(copies, copies.shape[1:], stream, out_dtype or torch.float32)
    st = lib().ab_group_average(_ptr(copies), copies.stride(0) if K > 1 else count, K, count, _dt(copies), _dt(out),
                                _ptr(out), _stream(stream))
    _check(st, "ab_group_average")
    return out


def ab_recombine(Abar, Bbar, W=None, ws=None, stream=None):
    """W = Abar Bbar in fp32."""
    _dev_ok(Abar, Bbar, W)
    m, r = Abar.shape
    n = Bbar.shape[1]
    if W is None:
        W = _result(Abar, (m, n), stream, torch.float32)
    if ws is None:
        ws = _scratch(ab_workspace_bytes(AB_OP_RECOMBINE, 0, m, n, r, 1, _dt(Abar)), Abar.device, stream)
    st = lib().ab_recombine(_ptr(Abar), _ptr(Bbar), _ptr(W), m, n, r, Abar.stride(0), Bbar.stride(0), _dt(Abar),
                            _ptr(ws), ws.numel(), _stream(stream))
    _check(st, "ab_recombine")
    return W


def ab_recombine_mean(A_copies, B_copies, W=None, Abar=None, Bbar=None, want_means=True, stream=None):
    """W = mean_k(A_k) mean_k(B_k) in one kernel; A_copies (K, m, r), B_copies (K, r, n), fp32.
    Returns (W, Abar, Bbar) (the means are None when want_means is False and none were passed)."""
    _dev_ok(A_copies, B_copies, W, Abar, Bbar)
    K, m, r = A_copies.shape
    n = B_copies.shape[2]
    if W is None:
        W = _result(A_copies, (m, n), stream, torch.float32)
    if want_means and Abar is None:
        Abar = _result(A_copies, (m, r), stream, torch.float32)
    if want_means and Bbar is None:
        Bbar = _result(A_copies, (r, n), stream, torch.float32)
    st = lib().ab_recombine_mean(_ptr(A_copies), A_copies.stride(0) if K > 1 else m * r, _ptr(B_copies),
                                 B_copies.stride(0) if K > 1 else r * n, K, _ptr(W), _ptr(Abar), _ptr(Bbar), m, n, r,
                                 _dt(A_copies), _stream(stream))
    _check(st, "ab_recombine_mean")
    return W, Abar, Bbar


def ab_svd_split(W, r_max, sigma_cutoff=0.0, out_dtype=None, ws=None, stream=None):
    """A = U_r' S^(1/2), B = S^(1/2) V_r'^T under the rank rule.  Returns (A, B, sigma, r_out, dev_status);
    r_out and dev_status are device int tensors (read them after synchronising)."""
    _dev_ok(W)
    m, n = W.shape
    od = out_dtype or W.dtype
    r_cap = min(r_max, m, n)
    A = _result(W, (m, r_max), stream, od)
    B = _result(W, (r_max, n), stream, od)
    sigma = _result(W, (r_cap,), stream, torch.float32)
    r_out = _result(W, (1,), stream, torch.int32, zero=True)
    status = _result(W, (1,), stream, torch.int32, zero=True)
    if ws is None:
        ws = _scratch(ab_workspace_bytes(AB_OP_SVD_SPLIT, 0, m, n, r_max, 1, _dt(W)), W.device, stream)
    st = lib().ab_svd_split(_ptr(W), m, n, r_max, float(sigma_cutoff), _ptr(A), _ptr(B), _ptr(sigma), _ptr(r_out),
                            _ptr(status), _dt(W), AB_BF16 if od == torch.bfloat16 else AB_F32, _ptr(ws), ws.numel(),
                            _stream(stream))
    _check(st, "ab_svd_split")
    return A, B, sigma, r_out, status


class SyncPlan:
    """Buffers and descriptors of one model's group synchronisation (ab_group_sync).  The buffers belong to the stream that the plan is made
    on: another one that runs the call waits for that first, and the plan stays until it has run it."""

    def __init__(self, A_copies, B_copies, sigma_cutoff, want_W=False, strided=False):
        """A_copies[i]: (K, m, r), B_copies[i]: (K, r, n).  strided=True accepts views whose copies are
        each contiguous but spaced by any stride along the leading axis (e.g. slices of a packed arena)."""
        self.A_copies, self.B_copies = list(A_copies), list(B_copies)
        self.L = len(self.A_copies)
        self.K = self.A_copies[0].shape[0]
        self.cutoff = float(sigma_cutoff)
        dev = self.A_copies[0].device
        self.dt = _dt(self.A_copies[0])
        self.A_out, self.B_out, self.sigma, self.W_out = [], [], [], []
        self.r_out = torch.zeros((self.L,), dtype=torch.int32, device=dev)
        self.status = torch.zeros((self.L,), dtype=torch.int32, device=dev)
        self.descs = (ab_sync_desc * self.L)()
        for i, (Ak, Bk) in enumerate(zip(self.A_copies, self.B_copies)):
            if strided:
                if not (Ak.is_cuda and Bk.is_cuda and Ak[0].is_contiguous() and Bk[0].is_contiguous()):
                    raise ValueError("each copy must be a contiguous CUDA tensor")
            else:
                _dev_ok(Ak, Bk)
            K, m, r = Ak.shape
            n = Bk.shape[2]
            self.A_out.append(torch.empty((m, r), dtype=Ak.dtype, device=dev))
            self.B_out.append(torch.empty((r, n), dtype=Ak.dtype, device=dev))
            self.sigma.append(torch.empty((min(r, m, n),), dtype=torch.float32, device=dev))
            d = self.descs[i]
            d.A_copies, d.B_copies = Ak.data_ptr(), Bk.data_ptr()
            d.strideA, d.strideB = (Ak.stride(0), Bk.stride(0)) if K > 1 else (m * r, r * n)
            d.m, d.n, d.r = m, n, r
            d.A_out, d.B_out = self.A_out[i].data_ptr(), self.B_out[i].data_ptr()
            d.sigma = self.sigma[i].data_ptr()
            d.r_out = self.r_out.data_ptr() + 4 * i
            if want_W:
                self.W_out.append(torch.empty((m, n), dtype=torch.float32, device=dev))
                d.W_out = self.W_out[i].data_ptr()
            else:
                d.W_out = None
        self.ws = workspace(lib().ab_sync_workspace_bytes(self.descs, self.L, self.K, self.dt), dev)


def ab_group_sync(plan: SyncPlan, stream=None, path=AB_SYNC_AUTO):
    """Mean of K copies -> W = Abar Bbar -> split under the rank rule, for every matrix of the plan.
    path: AB_SYNC_AUTO / AB_SYNC_DENSE (forms W, dense split) / AB_SYNC_FACTORED (r x r problems only)."""
    st = lib().ab_group_sync(plan.descs, plan.L, plan.K, plan.cutoff, plan.dt, _ptr(plan.status), _ptr(plan.ws),
                             plan.ws.numel(), _stream(stream), int(path))
    _check(st, "ab_group_sync")
    return plan.A_out, plan.B_out, plan.sigma, plan.r_out, plan.status
