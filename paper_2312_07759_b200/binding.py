"""Thin ctypes binding of the C-ABI library ``libidkm.so`` (see ``include/idkm.h``).

Argument marshalling only: every step of the path runs in the library's CUDA kernels.  PyTorch
supplies device memory (``tensor.data_ptr()``) and the current stream.  Importing this module
raises if the library has not been built; there is no CPU fallback.

Calls take a ``stream``.  Those on codes with group scales and on logits (``assign_groups``, ``matmul_codes``,
``distill_*``) mark their tensors as used on it; for the others, and for a ``Context``'s, the caller keeps the
tensors of a call until that stream is past it.
"""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass
from typing import List, Optional, Sequence

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libidkm.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2312_07759_b200.build` "
                      "(nvcc, sm_100a).  There is no fallback path.")
lib = C.CDLL(LIB_PATH)

IMPLICIT, JFB = 0, 1
OK, MAXITER = 0, 1
ERR_NULL, ERR_ALIGN, ERR_SHAPE, ERR_UNSUPPORTED, ERR_PARAM = -1, -2, -3, -4, -5
ERR_WORKSPACE, ERR_ORDER, ERR_CUDA, ERR_NONFINITE, ERR_DIVERGED = -6, -7, -8, -9, -10
ERR_NOALLOC_TOO_LARGE, ERR_TIMEOUT = -11, -12


class Info(C.Structure):
    _fields_ = [("status", C.c_int32), ("fwd_iters", C.c_int32), ("fwd_residual", C.c_float),
                ("dead_clusters", C.c_int32), ("adj_iters", C.c_int32), ("adj_residual", C.c_float)]

    def __repr__(self):
        return (f"Info(status={self.status}, fwd_iters={self.fwd_iters}, fwd_residual={self.fwd_residual:.3e}, "
                f"dead={self.dead_clusters}, adj_iters={self.adj_iters}, adj_residual={self.adj_residual:.3e})")


_vp, _i64p, _fp = C.c_void_p, C.POINTER(C.c_int64), C.c_void_p
lib.idkm_create.argtypes = [C.POINTER(_vp)]
lib.idkm_create.restype = C.c_int
lib.idkm_destroy.argtypes = [_vp]
lib.idkm_destroy.restype = None
lib.idkm_workspace_bytes.argtypes = [C.c_int64, C.c_int, C.c_int, C.c_int]
lib.idkm_workspace_bytes.restype = C.c_size_t
lib.idkm_forward.argtypes = [_vp, _fp, C.c_int64, C.c_int, _fp, C.c_int, C.c_float, C.c_float, C.c_int, _fp, _fp, _fp,
                             _vp, C.c_size_t, _vp]
lib.idkm_forward.restype = C.c_int
lib.idkm_forward_batched.argtypes = [_vp, _fp, _i64p, C.c_int, C.c_int, _fp, C.c_int, C.c_float, C.c_float, C.c_int,
                                     _fp, _fp, _fp, _vp, C.c_size_t, _vp]
lib.idkm_forward_batched.restype = C.c_int
lib.idkm_backward.argtypes = [_vp, _fp, C.c_int, C.c_float, C.c_int, C.c_float, _fp, _fp, _vp, C.c_size_t, _vp]
lib.idkm_backward.restype = C.c_int
lib.idkm_backward_restart.argtypes = [_vp, _fp, C.c_float, C.c_int, C.c_float, C.c_int, _fp, _fp, _vp, C.c_size_t, _vp,
                                      C.POINTER(C.c_float), C.POINTER(C.c_int)]
lib.idkm_backward_restart.restype = C.c_int
lib.idkm_get_info.argtypes = [_vp, C.POINTER(Info)]
lib.idkm_get_info.restype = C.c_int
lib.idkm_quantize_host.argtypes = [_vp, _fp, _i64p, C.c_int, C.c_int, _fp, C.c_int, C.c_float, C.c_float, C.c_int,
                                   _fp, C.c_int, C.c_float, C.c_int, C.c_float, _fp, _fp, _fp, _fp, C.POINTER(Info)]
lib.idkm_quantize_host.restype = C.c_int
lib.idkm_quantize_host_ex.argtypes = [_vp, _fp, _i64p, C.c_int, C.c_int, _fp, C.c_int, C.c_float, C.c_float, C.c_int,
                                      _fp, C.c_int, C.c_float, C.c_int, C.c_float, _fp, _fp, _fp, _fp, _fp, _fp,
                                      C.POINTER(Info)]
lib.idkm_quantize_host_ex.restype = C.c_int
lib.idkm_set_timing.argtypes = [_vp, C.c_int]
lib.idkm_set_timing.restype = C.c_int
lib.idkm_get_phase_ms.argtypes = [_vp, C.POINTER(C.c_float)]
lib.idkm_get_phase_ms.restype = C.c_int
lib.idkm_step_noalloc.argtypes = [_fp, C.c_int64, C.c_int, _fp, C.c_int, C.c_float, _fp, _vp]
lib.idkm_step_noalloc.restype = C.c_int
lib.idkm_step_noalloc_status.argtypes = [C.POINTER(C.c_int), _vp]
lib.idkm_step_noalloc_status.restype = C.c_int
lib.idkm_set_test_hooks.argtypes = [_vp, C.c_int, C.c_int64]
lib.idkm_set_test_hooks.restype = C.c_int
lib.idkm_count_busy_tickets.argtypes = [_vp, C.POINTER(C.c_int)]
lib.idkm_count_busy_tickets.restype = C.c_int
lib.idkm_set_wq_dtype.argtypes = [_vp, C.c_int]
lib.idkm_set_wq_dtype.restype = C.c_int
lib.idkm_set_collapse_step.argtypes = [_vp, C.c_int]
lib.idkm_set_collapse_step.restype = C.c_int
lib.idkm_set_distance.argtypes = [_vp, C.c_int]
lib.idkm_set_distance.restype = C.c_int
lib.idkm_set_adjoint_method.argtypes = [_vp, C.c_int]
lib.idkm_set_adjoint_method.restype = C.c_int
lib.idkm_get_history.argtypes = [_vp, C.c_int, C.c_int, C.POINTER(C.c_float), C.c_int, C.POINTER(C.c_int)]
lib.idkm_get_history.restype = C.c_int
lib.idkm_set_forward_loop.argtypes = [_vp, C.c_int]
lib.idkm_set_forward_loop.restype = C.c_int
lib.idkm_describe_path.argtypes = [C.c_int, C.c_int, C.c_int, C.c_int, C.POINTER(C.c_int)]
lib.idkm_describe_path.restype = C.c_int
lib.idkm_last_route.argtypes = [_vp, C.POINTER(C.c_int), C.POINTER(C.c_int)]
lib.idkm_last_route.restype = C.c_int
lib.idkm_launch_count.argtypes = [_vp]
lib.idkm_launch_count.restype = C.c_int64
lib.idkm_measure_pipe_rates.argtypes = [C.POINTER(C.c_double), C.POINTER(C.c_double), _vp]
lib.idkm_measure_pipe_rates.restype = C.c_int
lib.idkm_assign.argtypes = [_fp, C.c_int64, C.c_int, _fp, C.c_int, _vp, _fp, _vp]
lib.idkm_assign.restype = C.c_int
lib.idkm_code_bits.argtypes = [C.c_int]
lib.idkm_code_bits.restype = C.c_int
lib.idkm_codes_bytes.argtypes = [C.c_int64, C.c_int]
lib.idkm_codes_bytes.restype = C.c_size_t
lib.idkm_group_codes_pitch.argtypes = [C.c_int64]
lib.idkm_group_codes_pitch.restype = C.c_int64
lib.idkm_assign_groups.argtypes = [_vp, C.c_int, C.c_int64, C.c_int64, C.c_int64, _vp, C.c_int, C.c_int, C.c_int64, _vp, _vp, _vp, _vp]
lib.idkm_assign_groups.restype = C.c_int
lib.idkm_matmul_codes.argtypes = [_vp, C.c_int, C.c_int64, C.c_int64, _vp, C.c_int64, C.c_int64, C.c_int64, _vp, C.c_int, _vp, C.c_int64,
                                  _vp, C.c_int64, _vp]
lib.idkm_matmul_codes.restype = C.c_int
lib.idkm_set_codes_test_hooks.argtypes = [C.c_int]
lib.idkm_set_codes_test_hooks.restype = C.c_int
_logits = [_vp, C.c_int, C.c_int64, C.c_int64, C.c_int64, _vp, C.c_int, _vp, C.c_int, C.c_int, C.c_float]
lib.idkm_distill_forward.argtypes = _logits + [_vp, _vp, _vp]
lib.idkm_distill_forward.restype = C.c_int
lib.idkm_distill_backward.argtypes = _logits + [_vp, _vp, _vp, C.c_int64, _vp]
lib.idkm_distill_backward.restype = C.c_int
lib.idkm_distill_step.argtypes = _logits + [_vp, _vp, _vp, C.c_int64, _vp]
lib.idkm_distill_step.restype = C.c_int
lib.idkm_status_string.argtypes = [C.c_int]
lib.idkm_status_string.restype = C.c_char_p


class IdkmError(RuntimeError):
    def __init__(self, code: int):
        self.code = code
        super().__init__(f"idkm status {code}: {status_string(code)}")


def status_string(code: int) -> str:
    return lib.idkm_status_string(int(code)).decode()


def _check(rc: int) -> None:
    if rc != OK:
        raise IdkmError(rc)


def workspace_bytes(m_total: int, d: int, k: int, n_layers: int = 1) -> int:
    return int(lib.idkm_workspace_bytes(int(m_total), int(d), int(k), int(n_layers)))


def _ptr(t) -> Optional[int]:
    return None if t is None else int(t.data_ptr())


def _stream(stream) -> Optional[int]:
    if stream is None:
        import torch
        stream = torch.cuda.current_stream()
    h = int(stream.cuda_stream) if hasattr(stream, "cuda_stream") else int(stream)
    return h if h != 0 else None


@dataclass
class ForwardResult:
    C: "object"          # torch [L*k, d]
    Wq: "object"         # torch [m, d] or None
    A: "object"          # torch [m, k] or None


def step_noalloc(W, C_in, tau: float, C_out=None, stream=None):
    """``idkm_step_noalloc``: C_out = F(C_in, W) on CUDA tensors without any allocation inside the library.
    The caller passes C_out to keep the call itself allocation-free; if omitted it is created here, by torch."""
    import torch
    assert W.is_cuda and C_in.is_cuda and W.dtype == torch.float32 and W.is_contiguous() and C_in.is_contiguous()
    if C_out is None:
        C_out = torch.empty_like(C_in)
    _check(lib.idkm_step_noalloc(_ptr(W), int(W.shape[0]), int(W.shape[1]), _ptr(C_in), int(C_in.shape[0]),
                                 float(tau), _ptr(C_out), _stream(stream)))
    return C_out


def step_noalloc_status(stream=None) -> int:
    """``idkm_step_noalloc_status``: the device-side status of the last ``step_noalloc`` on the current device."""
    st = C.c_int(0)
    _check(lib.idkm_step_noalloc_status(C.byref(st), _stream(stream)))
    return int(st.value)


def assign(W, Cm, want_codes: bool = True, want_Wq: bool = True, stream=None):
    """``idkm_assign``: packed nearest-centroid codes (uint8 CUDA tensor) and dequantised weights of CUDA fp32 W."""
    import torch
    assert W.is_cuda and Cm.is_cuda and W.dtype == torch.float32 and Cm.dtype == torch.float32
    assert W.is_contiguous() and Cm.is_contiguous() and W.shape[1] == Cm.shape[1]
    m, d, k = int(W.shape[0]), int(W.shape[1]), int(Cm.shape[0])
    codes = torch.empty(int(lib.idkm_codes_bytes(m, k)), dtype=torch.uint8, device=W.device) if want_codes else None
    Wq = torch.empty_like(W) if want_Wq else None
    _check(lib.idkm_assign(_ptr(W), m, d, _ptr(Cm), k, _ptr(codes) if codes is not None else None,
                           _ptr(Wq) if Wq is not None else None, _stream(stream)))
    return codes, Wq


_ELEM = {}   # element types by torch's names for them, as idkm_set_wq_dtype numbers them


def _elem(t) -> int:
    """The number of a tensor's element type."""
    e = _ELEM.get(t.dtype)
    if e is None:
        if not _ELEM:
            import torch
            _ELEM.update({torch.float32: 0, torch.bfloat16: 1, torch.float16: 2})
            return _elem(t)
        raise IdkmError(ERR_UNSUPPORTED)
    return e


def _matrix(t):
    """(rows, columns, elements between rows) of a matrix whose rows are contiguous."""
    shape, stride = t.shape, t.stride()
    if len(shape) != 2 or (stride[1] != 1 and shape[1] > 1):
        raise ValueError(f"a matrix with contiguous rows expected, not shape {tuple(shape)} with strides {stride}")
    return shape[0], shape[1], stride[0] if shape[0] > 1 else shape[1]


class _Place:
    """Where a call runs that does not run on the current stream of the current device: inside the ``with`` that device is
    current, and new tensors belong to that stream.  ``given``: the stream, if one was given."""
    __slots__ = ("handle", "given", "_with")

    def __init__(self, stream, dev):
        import torch
        self.given = None
        if stream is None:
            self._with = torch.cuda.device(dev)
            self.handle = torch.cuda.current_stream(dev).cuda_stream or None
            return
        if not hasattr(stream, "cuda_stream"):
            stream = torch.cuda.ExternalStream(int(stream), device=dev)
        if stream.device.index != dev:
            raise ValueError(f"a stream of device {dev} expected, not of {stream.device}")
        self.given = stream
        self._with = torch.cuda.stream(stream)
        self.handle = int(stream.cuda_stream) or None

    def __enter__(self):
        self._with.__enter__()
        return self

    def __exit__(self, *a):
        self._with.__exit__(*a)


def _run(stream, call, first, *others):
    """``call(stream handle)`` on the device of the tensors, which have to be on one, and on ``stream``, or that device's current
    one.  (A call on the current device's current stream, the usual case, costs no context manager.)  The memory of the tensors
    is not handed out again before a given stream is past the call, even if the caller lets go of them right after it."""
    import torch
    dev = first.get_device()
    if dev < 0:
        raise ValueError("tensors on a CUDA device expected")
    for o in others:
        if o is not None and o.get_device() != dev:
            raise ValueError(f"tensors on one device expected: {first.device} and {o.device}")
    if stream is None and torch._C._cuda_getDevice() == dev:
        return call(torch._C._cuda_getCurrentRawStream(dev) or None)
    with _Place(stream, dev) as at:
        made = call(at.handle)
    if at.given is not None:
        for t in (first, *others):
            if t is not None:
                t.record_stream(at.given)
    return made


def _apart(out, *inputs) -> None:
    """A given output may not share memory with an input (rows of either may lie between the other's)."""
    base, rows = out.untyped_storage().data_ptr(), None
    for t in inputs:
        if t is not None and t.untyped_storage().data_ptr() == base and t.numel():
            if rows is None:
                rows = _rows(out)
            if _meet(rows, _rows(t)):
                raise ValueError("the output shares memory with an input")


def _rows(t):
    """(first byte, rows, bytes from one to the next, bytes of one) of a tensor whose rows are contiguous."""
    size, at = t.element_size(), t.data_ptr()
    if t.is_contiguous():
        return at, 1, 1, t.numel() * size
    rows, cols, ld = _matrix(t)
    return at, rows, max(ld * size, 1), cols * size


def _meet(x, y) -> bool:
    """Whether a byte of x's rows is one of y's."""
    (a, n, p, u), (b, m, q, v) = x, y
    if a + (n - 1) * p + u <= b or b + (m - 1) * q + v <= a:
        return False
    if n > m:
        (a, n, p, u), (b, m, q, v) = y, x
    if p == q:   # only the difference of two rows' numbers counts: one row of x, and as many of y as there are differences
        b, m, n = b - (n - 1) * q, m + n - 1, 1
    for i in range(n):   # rows j of y with b + j q < end of x's row and b + j q + v > its beginning
        at = a + i * p
        if max(0, (at - v - b) // q + 1) <= min(m - 1, (at + u - 1 - b) // q):
            return True
    return False


def assign_groups(W, Cm, group: int, want_Wq: bool = False, stream=None):
    """``idkm_assign_groups``: 4-bit codes (uint8 [rows, 16 ceil(cols / 32)]), scales ([rows, ceil(cols / group)], of the type of
    the codebook ``Cm``) and, if wanted, the dequantised weights (of W's type) of a CUDA matrix W; ``Cm`` holds k <= 16 entries."""
    e, ew, (rows, cols, ld) = _elem(Cm), _elem(W), _matrix(W)
    if not Cm.is_contiguous() or group < 1:
        raise ValueError("a contiguous codebook and a positive group expected")

    def call(handle):
        import torch
        codes = torch.empty((rows, (cols + 31) // 32 * 16), dtype=torch.uint8, device=W.device)
        scales = Cm.new_empty((rows, -(-cols // group)))
        Wq = W.new_empty((rows, cols)) if want_Wq else None
        return codes, scales, Wq, lib.idkm_assign_groups(W.data_ptr(), ew, rows, cols, ld, Cm.data_ptr(), Cm.numel(), e, group, codes.data_ptr(),
                                                         scales.data_ptr(), Wq.data_ptr() if want_Wq else None, handle)

    codes, scales, Wq, rc = _run(stream, call, W, Cm)
    if rc:
        raise IdkmError(rc)
    return codes, scales, Wq


def matmul_codes(X, codes, Cm, scales=None, group: int = 0, out=None, stream=None):
    """``idkm_matmul_codes``: X [tokens, cols] times the transpose of the weights that ``codes`` ([rows, bytes], uint8, as
    ``assign_groups`` gives them; those of ``assign`` reshaped to rows) stand for with the codebook ``Cm`` and ``scales``
    ([rows, ceil(cols / group)], or None); returns [tokens, rows] of X's type, which is that of the codebook and the scales."""
    e, (tokens, cols, ldx), (rows, bytes_, pitch) = _elem(X), _matrix(X), _matrix(codes)
    if Cm.dtype != X.dtype or (scales is not None and scales.dtype != X.dtype):
        raise ValueError("X, codebook and scales of one element type expected")
    import torch
    if codes.dtype is not torch.uint8 or 2 * bytes_ < cols or not Cm.is_contiguous():
        raise ValueError("uint8 codes of at least cols / 2 bytes a row and a contiguous codebook expected")
    if scales is not None and (group < 1 or scales.shape != (rows, -(-cols // group)) or not scales.is_contiguous()):
        raise ValueError(f"contiguous scales of shape ({rows}, cols / group) expected")
    if bytes_ < (cols + 31) // 32 * 16:
        raise IdkmError(ERR_SHAPE)
    ldy = rows
    if out is not None:
        if out.shape != (tokens, rows) or out.dtype != X.dtype or out.device != X.device:
            raise ValueError(f"an output of shape ({tokens}, {rows}) and of X's type and device expected")
        ldy = _matrix(out)[2]
        _apart(out, X, codes, Cm, scales)

    def call(handle):
        Y = X.new_empty((tokens, rows)) if out is None else out
        return Y, lib.idkm_matmul_codes(X.data_ptr(), e, tokens, ldx, codes.data_ptr(), rows, cols, pitch, Cm.data_ptr(), Cm.numel(),
                                        None if scales is None else scales.data_ptr(), group, Y.data_ptr(), ldy, handle)

    Y, rc = _run(stream, call, X, codes, Cm, scales, out)
    if rc:
        raise IdkmError(rc)
    return Y


def set_codes_test_hooks(missing_copy: int = 0) -> None:
    """``idkm_set_codes_test_hooks`` (host-side fault injection for ``matmul_codes``; 0 restores production behaviour)."""
    _check(lib.idkm_set_codes_test_hooks(missing_copy))


def _distill_inputs(z, idx, t, tau):
    import torch
    rows, vocab, ld = _matrix(z)
    shape, size = idx.shape, idx.element_size()
    if idx.dtype is not torch.int64 and idx.dtype is not torch.int32:
        raise ValueError("indices of 32 or 64 bits expected")
    if len(shape) != 2 or shape != t.shape or shape[0] != rows or not idx.is_contiguous() or not t.is_contiguous():
        raise ValueError("contiguous indices and logits of the teacher of one shape (rows, top) expected")
    return z.data_ptr(), _elem(z), rows, vocab, ld, idx.data_ptr(), size, t.data_ptr(), _elem(t), shape[1], tau


def _row_weights(weight, rows):
    """The address of the rows' weights, or None."""
    if weight is None:
        return None
    import torch
    if weight.dtype is not torch.float32 or weight.shape != (rows,) or not weight.is_contiguous():
        raise ValueError(f"weight: contiguous float32 of shape ({rows},) expected")
    return weight.data_ptr()


def _distill_out(z, out, *inputs):
    """Elements between the rows of the gradient."""
    if out is None:
        return z.shape[1]
    if out.shape != z.shape or out.dtype != z.dtype or out.device != z.device:
        raise ValueError("an output of z's shape, type and device expected")
    ld = _matrix(out)[2]
    _apart(out, *inputs)
    if out.data_ptr() != z.data_ptr() or ld != _matrix(z)[2]:
        _apart(out, z)
    return ld


def distill_forward(z, idx, t, tau: float, stream=None):
    """``idkm_distill_forward``: (loss [rows], statistics [rows, 2] for ``distill_backward``), both float32, of the student's logits
    z [rows, vocab] against the teacher's logits t [rows, top] at the indices idx [rows, top] (int32 or int64; -1: no entry)."""
    a = _distill_inputs(z, idx, t, tau)

    def call(handle):
        import torch
        loss = torch.empty(a[2], dtype=torch.float32, device=z.device)
        stats = loss.new_empty((a[2], 2))
        return loss, stats, lib.idkm_distill_forward(*a, loss.data_ptr(), stats.data_ptr(), handle)

    loss, stats, rc = _run(stream, call, z, idx, t)
    if rc:
        raise IdkmError(rc)
    return loss, stats


def distill_backward(z, idx, t, tau: float, stats, weight=None, out=None, stream=None):
    """``idkm_distill_backward``: the gradient with respect to z ([rows, vocab], of z's type), rows weighted by ``weight`` (float32
    [rows], dL/dloss; None: 1), from the statistics of ``distill_forward``.  ``out`` may be z itself."""
    import torch
    a = _distill_inputs(z, idx, t, tau)
    w = _row_weights(weight, a[2])
    if stats.dtype is not torch.float32 or stats.shape != (a[2], 2) or not stats.is_contiguous():
        raise ValueError("the statistics of distill_forward expected")
    ld = _distill_out(z, out, idx, t, stats, weight)

    def call(handle):
        dz = z.new_empty((a[2], a[3])) if out is None else out
        return dz, lib.idkm_distill_backward(*a, stats.data_ptr(), w, dz.data_ptr(), ld, handle)

    dz, rc = _run(stream, call, z, idx, t, stats, weight, out)
    if rc:
        raise IdkmError(rc)
    return dz


def distill_step(z, idx, t, tau: float, weight=None, out=None, stream=None):
    """``idkm_distill_step``: (loss [rows], gradient [rows, vocab]) in one launch.  ``out`` may be z itself."""
    a = _distill_inputs(z, idx, t, tau)
    w = _row_weights(weight, a[2])
    ld = _distill_out(z, out, idx, t, weight)

    def call(handle):
        import torch
        loss = torch.empty(a[2], dtype=torch.float32, device=z.device)
        dz = z.new_empty((a[2], a[3])) if out is None else out
        return loss, dz, lib.idkm_distill_step(*a, w, loss.data_ptr(), dz.data_ptr(), ld, handle)

    loss, dz, rc = _run(stream, call, z, idx, t, weight, out)
    if rc:
        raise IdkmError(rc)
    return loss, dz


def describe_path(d: int, k: int, adj_max_iter: int = 0, adjoint_method: int = 0) -> dict:
    """``idkm_describe_path``: the kernel layouts and the adjoint route the library picks for (d, k)."""
    out = (C.c_int * 5)()
    _check(lib.idkm_describe_path(int(d), int(k), int(adj_max_iter), int(adjoint_method), out))
    return {"step_layout": (out[0], out[1]), "adjoint_layout": (out[2], out[3]),
            "adjoint_route": ("fused passes", "explicit Jacobian in registers", "explicit Jacobian in tiles",
                              "exact solve on the explicit Jacobian")[out[4]]}


def measure_pipe_rates(stream=None):
    """``idkm_measure_pipe_rates``: (fp32 FMA lane-operations/s, special-function lane-operations/s) measured now."""
    a, b = C.c_double(0.0), C.c_double(0.0)
    _check(lib.idkm_measure_pipe_rates(C.byref(a), C.byref(b), _stream(stream)))
    return float(a.value), float(b.value)


class Context:
    """One ``idkm_ctx``: remembers the last forward so that ``backward`` can follow it."""

    def __init__(self):
        h = _vp()
        _check(lib.idkm_create(C.byref(h)))
        self._h = h
        self._ws = None
        self._keep = None
        self.n_layers = 0
        self._wq_dtype = 0

    def close(self):
        if getattr(self, "_h", None):
            lib.idkm_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- raw calls (pointers as ints; used by the error-path tests) ------------------------------
    def forward_raw(self, W, m, d, C0, k, tau, tol, max_iter, C_out, A_out, Wq_out, ws, ws_bytes, stream=None) -> int:
        return int(lib.idkm_forward(self._h, W, m, d, C0, k, tau, tol, max_iter, C_out, A_out, Wq_out, ws, ws_bytes,
                                    stream))

    def backward_raw(self, dWq, mode, adj_tol, adj_max_iter, alpha, dW_out, dC_out, ws, ws_bytes, stream=None) -> int:
        return int(lib.idkm_backward(self._h, dWq, mode, adj_tol, adj_max_iter, alpha, dW_out, dC_out, ws, ws_bytes,
                                     stream))

    # -- tensor-level calls ---------------------------------------------------------------------
    def forward(self, W, C0, tau: float, tol: float, max_iter: int, *, layer_offsets: Optional[Sequence[int]] = None,
                want_Wq: bool = True, want_A: bool = False, stream=None) -> ForwardResult:
        """``idkm_forward`` / ``idkm_forward_batched`` on CUDA tensors W [m, d], C0 [L*k, d] (float32, contiguous)."""
        import torch
        assert W.is_cuda and C0.is_cuda and W.dtype == torch.float32 and C0.dtype == torch.float32
        assert W.is_contiguous() and C0.is_contiguous()
        m, d = int(W.shape[0]), int(W.shape[1])
        if layer_offsets is None:
            layer_offsets = [0, m]
        L = len(layer_offsets) - 1
        k = int(C0.shape[0]) // L
        nbytes = workspace_bytes(m, d, k, L)
        if nbytes == 0:
            raise IdkmError(ERR_UNSUPPORTED)
        if self._ws is None or self._ws.numel() < nbytes or self._ws.device != W.device:
            self._ws = torch.empty(nbytes, dtype=torch.uint8, device=W.device)
        Cout = torch.empty_like(C0)
        wq_type = (torch.float32, torch.bfloat16, torch.float16)[self._wq_dtype]
        Wq = torch.empty(W.shape, dtype=wq_type, device=W.device) if want_Wq else None
        A = torch.empty((m, k), dtype=torch.float32, device=W.device) if want_A else None
        offs = (C.c_int64 * (L + 1))(*[int(x) for x in layer_offsets])
        rc = lib.idkm_forward_batched(self._h, _ptr(W), offs, L, d, _ptr(C0), k, float(tau), float(tol), int(max_iter),
                                      _ptr(Cout), _ptr(A), _ptr(Wq), _ptr(self._ws), self._ws.numel(), _stream(stream))
        _check(rc)
        self._keep = (W, Cout)   # the backward reads them
        self.n_layers = L
        self._shape = (m, d, k, L)
        return ForwardResult(Cout, Wq, A)

    def backward(self, dWq, mode: int = IMPLICIT, adj_tol: float = 0.0, adj_max_iter: int = 30, alpha: float = 1.0,
                 *, want_dW: bool = True, want_dC: bool = True, stream=None):
        """``idkm_backward``; returns (dW [m, d] or None, dC [L*k, d] or None)."""
        import torch
        assert dWq.is_cuda and dWq.dtype == torch.float32 and dWq.is_contiguous()
        if self._keep is None:
            raise IdkmError(ERR_ORDER)
        m, d, k, L = self._shape
        assert tuple(dWq.shape) == (m, d)
        dW = torch.empty_like(dWq) if want_dW else None
        dC = torch.empty((L * k, d), dtype=torch.float32, device=dWq.device) if want_dC else None
        rc = lib.idkm_backward(self._h, _ptr(dWq), int(mode), float(adj_tol), int(adj_max_iter), float(alpha), _ptr(dW),
                               _ptr(dC), _ptr(self._ws), self._ws.numel(), _stream(stream))
        _check(rc)
        return dW, dC

    def backward_restart(self, dWq, adj_tol: float, adj_max_iter: int, alpha0: float = 1.0, max_halvings: int = 4, *,
                         want_dW: bool = True, want_dC: bool = True, stream=None):
        """``idkm_backward_restart``; returns (dW or None, dC or None, alpha of the last attempt, attempts)."""
        import torch
        assert dWq.is_cuda and dWq.dtype == torch.float32 and dWq.is_contiguous()
        if self._keep is None:
            raise IdkmError(ERR_ORDER)
        m, d, k, L = self._shape
        dW = torch.empty_like(dWq) if want_dW else None
        dC = torch.empty((L * k, d), dtype=torch.float32, device=dWq.device) if want_dC else None
        al, att = C.c_float(0.0), C.c_int(0)
        _check(lib.idkm_backward_restart(self._h, _ptr(dWq), float(adj_tol), int(adj_max_iter), float(alpha0),
                                         int(max_halvings), _ptr(dW), _ptr(dC), _ptr(self._ws), self._ws.numel(),
                                         _stream(stream), C.byref(al), C.byref(att)))
        return dW, dC, float(al.value), int(att.value)

    def info(self) -> List[Info]:
        arr = (Info * max(1, self.n_layers))()
        _check(lib.idkm_get_info(self._h, arr))
        return list(arr)

    def quantize_host(self, W, C0, G, tau, tol, max_iter, mode=IMPLICIT, adj_tol=0.0, adj_max_iter=30, alpha=1.0,
                      layer_offsets=None, want_Wq=True, want_dW=True, out=None, also_jfb=False):
        """``idkm_quantize_host`` on HOST arrays (numpy float32, C-contiguous; pinned memory is the caller's choice).

        ``out`` may carry preallocated host arrays {"C", "Wq", "dW", "dC", "dW_jfb", "dC_jfb"} to write into.  With
        ``also_jfb`` (``idkm_quantize_host_ex``) the Jacobian-free gradients are computed from the same forward and
        returned as two more arrays after the info list."""
        import numpy as np
        m, d = W.shape
        if layer_offsets is None:
            layer_offsets = [0, m]
        L = len(layer_offsets) - 1
        k = C0.shape[0] // L
        out = {} if out is None else out
        Cout = out.get("C") if out.get("C") is not None else np.empty_like(C0)
        Wq = (out.get("Wq") if out.get("Wq") is not None else np.empty_like(W)) if want_Wq else None
        dW = (out.get("dW") if out.get("dW") is not None else np.empty_like(W)) if want_dW else None
        dC = out.get("dC") if out.get("dC") is not None else np.empty_like(C0)
        offs = (C.c_int64 * (L + 1))(*[int(x) for x in layer_offsets])
        infos = (Info * L)()
        hp = lambda a: None if a is None else a.ctypes.data
        if also_jfb:
            dWj = out.get("dW_jfb") if out.get("dW_jfb") is not None else np.empty_like(W)
            dCj = out.get("dC_jfb") if out.get("dC_jfb") is not None else np.empty_like(C0)
            rc = lib.idkm_quantize_host_ex(self._h, hp(W), offs, L, d, hp(C0), k, float(tau), float(tol), int(max_iter),
                                           hp(G), int(mode), float(adj_tol), int(adj_max_iter), float(alpha), hp(Cout),
                                           hp(Wq), hp(dW), hp(dC), hp(dWj), hp(dCj), infos)
            _check(rc)
            self.n_layers = L
            return Cout, Wq, dW, dC, list(infos), dWj, dCj
        rc = lib.idkm_quantize_host(self._h, hp(W), offs, L, d, hp(C0), k, float(tau), float(tol), int(max_iter), hp(G),
                                    int(mode), float(adj_tol), int(adj_max_iter), float(alpha), hp(Cout), hp(Wq), hp(dW),
                                    hp(dC), infos)
        _check(rc)
        self.n_layers = L
        return Cout, Wq, dW, dC, list(infos)

    def set_wq_dtype(self, dtype: int) -> None:
        """``idkm_set_wq_dtype``: 0 = Wq in fp32 (default), 1 = bfloat16, 2 = float16; ``forward`` then returns Wq as a
        tensor of that type."""
        _check(lib.idkm_set_wq_dtype(self._h, int(dtype)))
        self._wq_dtype = int(dtype)

    def set_collapse_step(self, method: int) -> None:
        """``idkm_set_collapse_step``: 0 = collapsing layers step in the fp32 increment form (default), 1 = in fp64."""
        _check(lib.idkm_set_collapse_step(self._h, int(method)))

    def set_distance(self, squared: bool) -> None:
        """``idkm_set_distance``: False = Euclidean distance in the softmax (Algorithm 1), True = its square."""
        _check(lib.idkm_set_distance(self._h, 1 if squared else 0))
        self._keep = None if squared != getattr(self, "_squared", False) else self._keep
        self._squared = bool(squared)

    def set_adjoint_method(self, method: int) -> None:
        """0: explicit Jacobian where k*d <= 64 (default); 1: always one fused pass per adjoint step; 2: exact solve
        on the explicit Jacobian where k*d <= 64."""
        _check(lib.idkm_set_adjoint_method(self._h, int(method)))

    def history(self, which: int = 0, layer: int = 0, capacity: int = 1024):
        """``idkm_get_history``: residuals of the last forward (which=0) or implicit backward (which=1) loop of a layer,
        as a float32 numpy array, first iteration first."""
        import numpy as np
        buf = (C.c_float * capacity)()
        n = C.c_int(0)
        _check(lib.idkm_get_history(self._h, int(which), int(layer), buf, int(capacity), C.byref(n)))
        return np.frombuffer(buf, dtype=np.float32, count=n.value).copy()

    def set_forward_loop(self, method: int) -> None:
        """0: small layers and batches of them run the whole forward loop in one cooperative launch (default); 1: a launch per iteration;
        2: a launch per iteration and never the kernel that steps fp32 and fp64 layers side by side; 3: as 2 with the
        rows of small-codebook layers streamed by bulk asynchronous copies."""
        _check(lib.idkm_set_forward_loop(self._h, int(method)))

    def set_test_hooks(self, missing_arrivals: int = 0, spin_limit_ticks: int = 0) -> None:
        """``idkm_set_test_hooks``: host-side fault injection for the timeout path; (0, 0) switches it off."""
        _check(lib.idkm_set_test_hooks(self._h, int(missing_arrivals), int(spin_limit_ticks)))

    def busy_tickets(self) -> int:
        """``idkm_count_busy_tickets``: arrival counters of the last forward's workspace that are not at rest."""
        n = C.c_int(0)
        _check(lib.idkm_count_busy_tickets(self._h, C.byref(n)))
        return int(n.value)

    def set_timing(self, enable: bool = True) -> None:
        _check(lib.idkm_set_timing(self._h, 1 if enable else 0))

    def phase_ms(self) -> dict:
        """Elapsed milliseconds per phase of the last forward / backward (``idkm_get_phase_ms``)."""
        arr = (C.c_float * 6)()
        _check(lib.idkm_get_phase_ms(self._h, arr))
        return dict(zip(("init", "steps", "final", "grad", "adjoint", "scatter"), [float(x) for x in arr]))

    def last_route(self) -> dict:
        """``idkm_last_route``: which kernels the last forward and the last backward took."""
        f, a = C.c_int(0), C.c_int(0)
        _check(lib.idkm_last_route(self._h, C.byref(f), C.byref(a)))
        return {"forward": ("a launch per iteration", "one-launch loop", "one-launch loop of larger codebooks", "interval form")[f.value],
                "adjoint": ("none", "fused passes", "explicit Jacobian in registers", "explicit Jacobian in tiles",
                            "exact solve on the explicit Jacobian", "explicit Jacobian from the tensor cores", "interval sums")[a.value + 1]}

    @property
    def launches(self) -> int:
        return int(lib.idkm_launch_count(self._h))
