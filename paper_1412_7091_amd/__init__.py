"""Exact large-sparse-target output layer on MI355X: Python binding.

Thin ctypes binding of the C ABI declared in include/lst.h.  The functions
below carry the same names as the C entry points and only marshal arguments:
torch tensors (device memory) become pointers, torch's current HIP stream
becomes the library's stream.  Every step of the computation runs in the HIP
kernels of liblst.so; there is no other code path.  If the library has not been
built, load_library() raises instead of falling back to anything.

Classes FactoredOutputLayer and NaiveOutputLayer wrap a state handle.  The
operators around the layers (dropout, the gated recurrence, ...) hold no handle:
they run on torch's current stream of their tensors' device, and their workspaces
are tensors of their own for each call.  Like the layers they take no part in
torch's autograd: forward and backward passes are called by name, and what comes
back from a tensor that requires a gradient has no graph.
"""
from __future__ import annotations

import ctypes
import functools
import os
from typing import Optional, Tuple

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "liblst.so")

LST_OK = 0
LST_EINVAL = -1
LST_EINDEX = -2
LST_ESINGULAR = -3
LST_ENOMEM = -4
LST_EHIP = -5
LST_ENONFINITE = -6
LST_ESTATE = -7
LST_ENOSCRATCH = -8

LST_LOSS_SQUARED = 0
LST_LOSS_SPHERICAL = 1
LST_LOSS_SPHERICAL_SHIFTED = 2

LST_F32 = 0
LST_BF16 = 1
LST_F16 = 2

LST_RECUR_CHUNK = 128

_LOSS = {"squared": LST_LOSS_SQUARED, "spherical": LST_LOSS_SPHERICAL,
         "spherical_shifted": LST_LOSS_SPHERICAL_SHIFTED}


class lst_config(ctypes.Structure):
    _fields_ = [
        ("loss", ctypes.c_int32),
        ("sph_eps", ctypes.c_float),
        ("m_max", ctypes.c_int32),
        ("K_max", ctypes.c_int32),
        ("cond_max", ctypes.c_float),
    ]


class lst_stats_t(ctypes.Structure):
    _fields_ = [
        ("steps", ctypes.c_int64),
        ("restores", ctypes.c_int64),
        ("last_unique", ctypes.c_int32),
        ("last_nnz", ctypes.c_int32),
    ]


class lst_stab_config(ctypes.Structure):
    _fields_ = [
        ("sigma_low", ctypes.c_float),
        ("sigma_high", ctypes.c_float),
        ("squarings", ctypes.c_int32),
        ("max_fixes", ctypes.c_int32),
        ("reinvert", ctypes.c_int32),
    ]


class lst_stab_report(ctypes.Structure):
    _fields_ = [
        ("fixes_low", ctypes.c_int32),
        ("fixes_high", ctypes.c_int32),
        ("sigma_min", ctypes.c_float),
        ("sigma_max", ctypes.c_float),
    ]


class LstError(RuntimeError):
    def __init__(self, code: int, what: str = ""):
        self.code = code
        msg = _lib.lst_strerror(code).decode() if _lib is not None else str(code)
        super().__init__(f"{what}: {msg} ({code})" if what else f"{msg} ({code})")


_lib: Optional[ctypes.CDLL] = None

_P = ctypes.c_void_p
_SIGS = {
    "lst_init": (ctypes.c_int, [ctypes.POINTER(_P), ctypes.c_int64, ctypes.c_int32, _P, _P,
                                ctypes.POINTER(lst_config), _P]),
    "lst_step": (ctypes.c_int, [_P, ctypes.c_int32, ctypes.c_int32, _P, _P, _P, ctypes.c_float,
                                _P, _P]),
    "lst_step_solve": (ctypes.c_int, [_P, ctypes.c_int32, ctypes.c_int32, _P, _P, _P,
                                      ctypes.c_float, _P, _P]),
    "lst_materialize_W": (ctypes.c_int, [_P, _P]),
    "lst_get_state": (ctypes.c_int, [_P, _P, _P, _P]),
    "lst_get_V": (ctypes.c_int, [_P, _P]),
    "lst_get_shift": (ctypes.c_int, [_P, _P, _P]),
    "lst_touched_rows": (ctypes.c_int, [_P, _P, ctypes.c_int32, ctypes.POINTER(ctypes.c_int32)]),
    "lst_restore": (ctypes.c_int, [_P]),
    "lst_stabilize": (ctypes.c_int, [_P, ctypes.POINTER(lst_stab_config),
                                     ctypes.POINTER(lst_stab_report)]),
    "lst_stabilize_noalloc": (ctypes.c_int, [_P, ctypes.POINTER(lst_stab_config),
                                             ctypes.POINTER(lst_stab_report)]),
    "lst_set_stabilize": (ctypes.c_int, [_P, ctypes.c_int32, ctypes.POINTER(lst_stab_config)]),
    "lst_naive_init": (ctypes.c_int, [ctypes.POINTER(_P), ctypes.c_int64, ctypes.c_int32, _P,
                                      ctypes.POINTER(lst_config), _P]),
    "lst_naive_step": (ctypes.c_int, [_P, ctypes.c_int32, ctypes.c_int32, _P, _P, _P,
                                      ctypes.c_float, _P, _P]),
    "lst_sync": (ctypes.c_int, [_P]),
    "lst_set_graphs": (ctypes.c_int, [_P, ctypes.c_int32]),
    "lst_set_split_tasks": (ctypes.c_int, [_P, ctypes.c_int32]),
    "lst_stats": (ctypes.c_int, [_P, ctypes.POINTER(lst_stats_t)]),
    "lst_profile_enable": (ctypes.c_int, [_P, ctypes.c_int32]),
    "lst_profile_read": (ctypes.c_int, [_P, ctypes.POINTER(ctypes.c_double), ctypes.c_int32,
                                        ctypes.POINTER(ctypes.c_int32),
                                        ctypes.POINTER(ctypes.c_int64)]),
    "lst_profile_phase_name": (ctypes.c_char_p, [ctypes.c_int32]),
    "lst_input_init": (ctypes.c_int, [ctypes.POINTER(_P), ctypes.c_int64, ctypes.c_int32, _P, _P]),
    "lst_input_forward": (ctypes.c_int, [_P, ctypes.c_int32, ctypes.c_int32, _P, _P, _P]),
    "lst_input_update": (ctypes.c_int, [_P, ctypes.c_int32, ctypes.c_int32, _P, _P, _P,
                                        ctypes.c_float]),
    "lst_input_get_W": (ctypes.c_int, [_P, _P]),
    "lst_input_sync": (ctypes.c_int, [_P]),
    "lst_input_free": (None, [_P]),
    "lst_dropout": (ctypes.c_int, [ctypes.c_int32, ctypes.c_int64, ctypes.c_int32, _P,
                                   ctypes.c_int64, _P, ctypes.c_int64, _P, ctypes.c_int64,
                                   ctypes.c_double, ctypes.c_uint64, ctypes.c_uint64, _P, _P]),
    "lst_recur_forward": (ctypes.c_int, [ctypes.c_int32] * 4 + [
        _P, ctypes.c_int64, _P, ctypes.c_int64, _P, _P, _P, ctypes.c_int64, _P, _P, _P, _P, _P]),
    "lst_recur_backward": (ctypes.c_int, [ctypes.c_int32] * 4 + [
        _P, ctypes.c_int64, _P, ctypes.c_int64, _P, _P, _P, ctypes.c_int64, _P, _P, _P,
        ctypes.c_int64, _P, ctypes.c_int64, _P, _P, _P, _P]),
    "lst_recur_saved": (ctypes.c_int64, [ctypes.c_int32, ctypes.c_int32]),
    "lst_recur_workspace": (ctypes.c_int64, [ctypes.c_int32, ctypes.c_int32]),
    "lst_recur_step": (ctypes.c_int, [ctypes.c_int32] * 4 + [
        _P, ctypes.c_int64, _P, ctypes.c_int64, _P, _P, _P, ctypes.c_int64, _P, _P]),
    "lst_quantize": (ctypes.c_int, [ctypes.c_int32, ctypes.c_int64, ctypes.c_int32, _P,
                                    ctypes.c_int64, _P, _P, _P]),
    "lst_scores_workspace": (ctypes.c_int64, [ctypes.c_int32, ctypes.c_int32]),
    "lst_scores": (ctypes.c_int, [ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_int64,
                                  ctypes.c_int32, _P, ctypes.c_int64, _P, _P, _P, ctypes.c_int64,
                                  _P, _P]),
    "lst_sample": (ctypes.c_int, [ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, _P,
                                  ctypes.c_int64, _P, _P, _P, _P, _P, _P, _P, _P, _P]),
    "lst_sample_workspace": (ctypes.c_int64, [ctypes.c_int32, ctypes.c_int32]),
    "lst_strerror": (ctypes.c_char_p, [ctypes.c_int]),
    "lst_free": (None, [_P]),
}

EXPORTED = tuple(_SIGS)


def load_library(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load liblst.so (once).  Raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(
            f"{path} not found: build the HIP library first (python -m paper_1412_7091_amd.build)")
    lib = ctypes.CDLL(path)
    for name, (res, args) in _SIGS.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _lib = lib
    return lib


def _check(code: int, what: str) -> None:
    if code != LST_OK:
        raise LstError(code, what)


def _ptr(t, dtype, what: str):
    """Device pointer of a contiguous CUDA tensor of the given dtype (None -> NULL)."""
    import torch

    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{what} must be a device tensor")
    if t.dtype != dtype:
        raise TypeError(f"{what} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous")
    return ctypes.c_void_p(t.data_ptr())


def _stream_handle(stream=None):
    import torch

    s = stream if stream is not None else torch.cuda.current_stream()
    return ctypes.c_void_p(s.cuda_stream)


def _config(loss: str, sph_eps: float, m_max: int, K_max: int, cond_max: float) -> lst_config:
    if loss not in _LOSS:
        raise ValueError(f"loss must be one of {sorted(_LOSS)}")
    return lst_config(_LOSS[loss], float(sph_eps), int(m_max), int(K_max), float(cond_max))


# ----------------------------------------------------------- C-named wrappers
def lst_init(V, U=None, *, loss="squared", sph_eps=1e-3, m_max=128, K_max=16, cond_max=0.0,
             stream=None):
    """Create a factored state from device tensors V (D x d) and U (d x d or None)."""
    import torch

    lib = load_library()
    D, d = V.shape
    cfg = _config(loss, sph_eps, m_max, K_max, cond_max)
    h = _P()
    _check(lib.lst_init(ctypes.byref(h), D, d, _ptr(V, torch.float32, "V"),
                        _ptr(U, torch.float32, "U"), ctypes.byref(cfg), _stream_handle(stream)),
           "lst_init")
    return h


def lst_naive_init(W, *, loss="squared", sph_eps=1e-3, m_max=128, K_max=16, stream=None):
    import torch

    lib = load_library()
    D, d = W.shape
    cfg = _config(loss, sph_eps, m_max, K_max, 0.0)
    h = _P()
    _check(lib.lst_naive_init(ctypes.byref(h), D, d, _ptr(W, torch.float32, "W"),
                              ctypes.byref(cfg), _stream_handle(stream)), "lst_naive_init")
    return h


def _step(fn_name, h, H, Y_idx, Y_val, lr, loss_out, grad_out):
    import torch

    m, d = H.shape
    K = Y_idx.shape[1]
    if Y_idx.shape[0] != m or (Y_val is not None and tuple(Y_val.shape) != tuple(Y_idx.shape)):
        raise ValueError("H, Y_idx and Y_val disagree on m / K")
    if tuple(loss_out.shape) != (m,) or tuple(grad_out.shape) != (m, d):
        raise ValueError("loss must be (m,) and grad_H (m, d)")
    fn = getattr(load_library(), fn_name)
    _check(fn(h, m, K, _ptr(H, torch.float32, "H"), _ptr(Y_idx, torch.int32, "Y_idx"),
              _ptr(Y_val, torch.float32, "Y_val"), float(lr),
              _ptr(loss_out, torch.float32, "loss"), _ptr(grad_out, torch.float32, "grad_H")),
           fn_name)


def lst_step(h, H, Y_idx, Y_val, lr, loss_out, grad_out):
    _step("lst_step", h, H, Y_idx, Y_val, lr, loss_out, grad_out)


def lst_step_solve(h, H, Y_idx, Y_val, lr, loss_out, grad_out):
    _step("lst_step_solve", h, H, Y_idx, Y_val, lr, loss_out, grad_out)


def lst_naive_step(h, H, Y_idx, Y_val, lr, loss_out, grad_out):
    _step("lst_naive_step", h, H, Y_idx, Y_val, lr, loss_out, grad_out)


def lst_materialize_W(h, W_out):
    import torch

    _check(load_library().lst_materialize_W(h, _ptr(W_out, torch.float32, "W")),
           "lst_materialize_W")


def lst_get_state(h, Q=None, U=None, UinvT=None):
    import torch

    _check(load_library().lst_get_state(h, _ptr(Q, torch.float32, "Q"),
                                        _ptr(U, torch.float32, "U"),
                                        _ptr(UinvT, torch.float32, "UinvT")), "lst_get_state")


def lst_get_V(h, V_out):
    import torch

    _check(load_library().lst_get_V(h, _ptr(V_out, torch.float32, "V")), "lst_get_V")


def lst_get_shift(h, c_out=None, s_out=None):
    import torch

    _check(load_library().lst_get_shift(h, _ptr(c_out, torch.float32, "c"),
                                        _ptr(s_out, torch.float32, "s")), "lst_get_shift")


def lst_touched_rows(h, capacity: int):
    import numpy as np

    buf = (ctypes.c_int32 * max(1, capacity))()
    n = ctypes.c_int32(0)
    _check(load_library().lst_touched_rows(h, buf, capacity, ctypes.byref(n)), "lst_touched_rows")
    return np.frombuffer(buf, dtype=np.int32, count=n.value).copy()


def lst_restore(h):
    _check(load_library().lst_restore(h), "lst_restore")


def _stab_config(sigma_low, sigma_high, squarings, max_fixes, reinvert) -> lst_stab_config:
    return lst_stab_config(float(sigma_low), float(sigma_high), int(squarings), int(max_fixes),
                           int(reinvert))


def lst_stabilize(h, sigma_low=1e-3, sigma_high=100.0, squarings=7, max_fixes=2, reinvert=1,
                  report=True):
    """Appendix C correction of out-of-range singular values of U.  With report, synchronises
    and returns the lst_stab_report; else enqueues and returns None."""
    cfg = _stab_config(sigma_low, sigma_high, squarings, max_fixes, reinvert)
    rep = lst_stab_report() if report else None
    _check(load_library().lst_stabilize(h, ctypes.byref(cfg),
                                        ctypes.byref(rep) if rep is not None else None),
           "lst_stabilize")
    return rep


def lst_stabilize_noalloc(h, sigma_low=1e-3, sigma_high=100.0, squarings=7, max_fixes=2,
                          reinvert=1, report=True):
    """lst_stabilize on the library's static workspace (no device allocation)."""
    cfg = _stab_config(sigma_low, sigma_high, squarings, max_fixes, reinvert)
    rep = lst_stab_report() if report else None
    _check(load_library().lst_stabilize_noalloc(h, ctypes.byref(cfg),
                                                ctypes.byref(rep) if rep is not None else None),
           "lst_stabilize_noalloc")
    return rep


def lst_set_stabilize(h, every, sigma_low=1e-3, sigma_high=100.0, squarings=7, max_fixes=2,
                      reinvert=1):
    cfg = _stab_config(sigma_low, sigma_high, squarings, max_fixes, reinvert)
    _check(load_library().lst_set_stabilize(h, int(every), ctypes.byref(cfg)),
           "lst_set_stabilize")


def lst_sync(h) -> int:
    """Wait for the state's stream; returns (and clears) the sticky device status code."""
    return int(load_library().lst_sync(h))


def lst_set_graphs(h, enable: bool = True) -> None:
    _check(load_library().lst_set_graphs(h, 1 if enable else 0), "lst_set_graphs")


def lst_set_split_tasks(h, enable: bool = True) -> None:
    _check(load_library().lst_set_split_tasks(h, 1 if enable else 0), "lst_set_split_tasks")


def lst_stats(h) -> lst_stats_t:
    st = lst_stats_t()
    _check(load_library().lst_stats(h, ctypes.byref(st)), "lst_stats")
    return st


def lst_profile_enable(h, enable: bool = True) -> None:
    _check(load_library().lst_profile_enable(h, 1 if enable else 0), "lst_profile_enable")


def lst_profile_read(h):
    """{phase name: summed milliseconds} over the profiled steps, and the step count."""
    lib = load_library()
    buf = (ctypes.c_double * 64)()
    n = ctypes.c_int32(0)
    steps = ctypes.c_int64(0)
    _check(lib.lst_profile_read(h, buf, 64, ctypes.byref(n), ctypes.byref(steps)),
           "lst_profile_read")
    return {lib.lst_profile_phase_name(i).decode(): buf[i] for i in range(n.value)}, steps.value


def lst_profile_phase_name(i: int):
    r = load_library().lst_profile_phase_name(i)
    return None if r is None else r.decode()


def lst_strerror(code: int) -> str:
    return load_library().lst_strerror(code).decode()


def lst_free(h) -> None:
    if h is not None and h.value:
        load_library().lst_free(h)


# ------------------------------------------- the operators around the layers
def _dtype_code(t, what: str) -> int:
    import torch

    code = {torch.float32: LST_F32, torch.bfloat16: LST_BF16, torch.float16: LST_F16}.get(t.dtype)
    if code is None:
        raise TypeError(f"{what} must be float32, bfloat16 or float16, got {t.dtype}")
    return code


def _matrix(t, what: str, like=None, shape=None):
    """Address and row stride of a device matrix with unit stride along its rows (None -> NULL);
    like: a tensor whose type and device it must have."""
    if t is None:
        return None, 0
    if not t.is_cuda:
        raise TypeError(f"{what} must be a device tensor")
    if t.dim() != 2 or (shape is not None and t.shape != shape):
        raise ValueError(f"{what} must be a matrix" + (f" of {tuple(shape)}" if shape else ""))
    if like is not None and (t.dtype != like.dtype or t.device != like.device):
        raise TypeError(f"{what} must be {like.dtype} on {like.device}, got {t.dtype} on {t.device}")
    rows, cols = t.shape
    ld = t.stride(0)
    if rows > 0x7FFFFFFF or cols > 0x7FFFFFFF:
        raise ValueError(f"{what} is too large")
    if rows <= 1:
        ld = cols
    if (cols > 1 and t.stride(1) != 1) or ld < cols:
        raise ValueError(f"{what} must have unit stride along its rows, and rows that do not overlap")
    return t.data_ptr(), ld


def _vector(t, dtype, what: str, device, count=None):
    """Address of a contiguous device tensor of the given type and number of elements."""
    if t is None:
        return None
    if not t.is_cuda or t.device != device:
        raise TypeError(f"{what} must be a tensor on {device}")
    if t.dtype != dtype:
        raise TypeError(f"{what} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous() or (count is not None and t.numel() != count):
        raise ValueError(f"{what} must be contiguous" +
                         (f" and hold {count} elements" if count is not None else ""))
    return t.data_ptr()


def _enqueue(name: str, device, *args) -> None:
    """Call an entry point with torch's current stream of the device as its last argument."""
    import torch

    fn = getattr(load_library(), name)
    # the handle alone: an object for it would take a sixth of a small call's time
    stream = torch._C._cuda_getCurrentRawStream(device.index)
    if device.index == torch.cuda.current_device():
        code = fn(*args, stream)
    else:
        with torch.cuda.device(device):
            code = fn(*args, stream)
    if code != LST_OK:
        raise LstError(code, name)


def _word(v, what: str) -> int:
    v = int(v)
    if not 0 <= v < 1 << 64:
        raise ValueError(f"{what} must be in [0, 2^64)")
    return v


def lst_dropout(x, p, seed, offset=0, *, residual=None, counter=None, out=None):
    """y = residual + x * keep / (1 - p); the mask is that of (seed, offset, row, column)."""
    import torch

    px, ldx = _matrix(x, "x")
    code = _dtype_code(x, "x")
    if out is None:
        out = x.new_empty(x.shape)
    pr, ldr = _matrix(residual, "residual", x, x.shape)
    py, ldy = _matrix(out, "out", x, x.shape)
    _enqueue("lst_dropout", x.device, code, x.shape[0], x.shape[1], px, ldx, pr, ldr, py, ldy,
             float(p), _word(seed, "seed"), _word(offset, "offset"),
             _vector(counter, torch.int64, "counter", x.device, 1))
    return out


@functools.lru_cache(maxsize=256)
def lst_recur_saved(rows: int, d: int) -> int:
    return int(load_library().lst_recur_saved(rows, d))


@functools.lru_cache(maxsize=256)
def lst_recur_workspace(rows: int, d: int) -> int:
    return int(load_library().lst_recur_workspace(rows, d))


def _recur_inputs(x, g, offsets, h0, n_seq):
    """Checked arguments that the forward and the backward pass share."""
    import torch

    px, ldx = _matrix(x, "x")
    code = _dtype_code(x, "x")
    pg, ldg = _matrix(g, "g", x, x.shape)
    if offsets is not None:
        if offsets.numel() < 1:
            raise ValueError("offsets must hold at least one element")
        have = offsets.numel() - 1
    elif n_seq is not None:
        have = int(n_seq)
    else:
        have = h0.shape[0] if h0 is not None else 1
    if n_seq is not None and n_seq != have:
        raise ValueError("n_seq and offsets disagree")
    if have > 1 << 30:
        raise ValueError("at most 2^30 sequences")
    rows, d = x.shape
    if h0 is not None and tuple(h0.shape) != (have, d):
        raise ValueError("h0 must be (n_seq, d)")
    if offsets is None and (have < 1 or rows % have):
        raise ValueError("without offsets, the rows must divide into n_seq equal sequences")
    return (have, (code, rows, have, d, px, ldx, pg, ldg,
                   _vector(offsets, torch.int32, "offsets", x.device),
                   _vector(h0, torch.float32, "h0", x.device)))


def _work(like, n: int):
    """n bytes of workspace beside a tensor, for one call (None for none)."""
    import torch

    return like.new_empty(n, dtype=torch.uint8) if n > 0 else None


def lst_recur_forward(x, g, offsets=None, h0=None, *, n_seq=None, out=None, h_last=None,
                      save=False, status=None):
    """(y, h_last, saved) of the gated recurrence; saved is None unless save."""
    import torch

    have, args = _recur_inputs(x, g, offsets, h0, n_seq)
    rows, d, dev = x.shape[0], x.shape[1], x.device
    if out is None:
        out = x.new_empty((rows, d))
    if h_last is None:
        h_last = x.new_empty((have, d), dtype=torch.float32)
    saved = None
    if save:
        saved = x.new_empty((max(lst_recur_saved(rows, d), 0) // max(d, 1), d),
                            dtype=torch.float32)
    work = _work(x, lst_recur_workspace(rows, d))
    _enqueue("lst_recur_forward", dev, *args, *_matrix(out, "out", x, x.shape),
             _vector(h_last, torch.float32, "h_last", dev, have * d),
             None if saved is None else saved.data_ptr(),
             None if work is None else work.data_ptr(),
             _vector(status, torch.int32, "status", dev, 1))
    return out, h_last, saved


def lst_recur_backward(x, g, grad_y, saved, offsets=None, h0=None, grad_last=None, *, n_seq=None,
                       out=None, status=None):
    """(grad_x, grad_g, grad_h0) from the forward pass' inputs and saved; out: the first two."""
    import torch

    have, args = _recur_inputs(x, g, offsets, h0, n_seq)
    rows, d, dev = x.shape[0], x.shape[1], x.device
    if out is None:
        out = x.new_empty((rows, d)), x.new_empty((rows, d))
    grad_h0 = x.new_empty((have, d), dtype=torch.float32)
    work = _work(x, lst_recur_workspace(rows, d))
    _enqueue("lst_recur_backward", dev, *args, *_matrix(grad_y, "grad_y", x, x.shape),
             _vector(grad_last, torch.float32, "grad_last", dev, have * d),
             _vector(saved, torch.float32, "saved", dev, lst_recur_saved(rows, d)),
             *_matrix(out[0], "grad_x", x, x.shape), *_matrix(out[1], "grad_g", x, x.shape),
             grad_h0.data_ptr(), None if work is None else work.data_ptr(),
             _vector(status, torch.int32, "status", dev, 1))
    return out[0], out[1], grad_h0


def lst_recur_step(x, g, h, slots=None, *, out=None, status=None):
    """One token for each row: h[slots[i]] moves on in place; returns the new states as y."""
    import torch

    px, ldx = _matrix(x, "x")
    code = _dtype_code(x, "x")
    pg, ldg = _matrix(g, "g", x, x.shape)
    rows, d, dev = x.shape[0], x.shape[1], x.device
    if h.dim() != 2 or h.shape[1] != d or h.shape[0] > 0x7FFFFFFF:
        raise ValueError("h must be (n_slots, d)")
    if out is None:
        out = x.new_empty((rows, d))
    _enqueue("lst_recur_step", dev, code, rows, h.shape[0], d, px, ldx, pg, ldg,
             _vector(slots, torch.int32, "slots", dev, rows),
             _vector(h, torch.float32, "h", dev), *_matrix(out, "out", x, x.shape),
             _vector(status, torch.int32, "status", dev, 1))
    return out


def lst_quantize(x, *, codes=None, scales=None):
    """(codes, scales) of a matrix in 8 bits, one scale for each block of 128 columns."""
    import torch

    px, ldx = _matrix(x, "x")
    code = _dtype_code(x, "x")
    rows, cols = x.shape
    blocks = (cols + 127) // 128
    if codes is None:
        codes = x.new_empty((rows, 128 * blocks), dtype=torch.uint8)
    if scales is None:
        scales = x.new_empty((rows, blocks), dtype=torch.uint8)
    _enqueue("lst_quantize", x.device, code, rows, cols, px, ldx,
             _vector(codes, torch.uint8, "codes", x.device, rows * 128 * blocks),
             _vector(scales, torch.uint8, "scales", x.device, rows * blocks))
    return codes, scales


@functools.lru_cache(maxsize=256)
def lst_scores_workspace(m: int, d: int) -> int:
    return int(load_library().lst_scores_workspace(m, d))


def lst_scores(H, codes, scales, *, dtype=None, out=None):
    """O = H W^T from the weights' codes and scales; dtype: that of O (H's when not given)."""
    import torch

    ph, ldh = _matrix(H, "H")
    code = _dtype_code(H, "H")
    (m, d), dev = H.shape, H.device
    D = scales.shape[0]
    blocks = (d + 127) // 128
    if scales.dim() != 2 or scales.shape[1] != blocks or codes.shape != (D, 128 * blocks):
        raise ValueError(f"codes and scales must be those of a matrix with {d} columns")
    if out is None:
        out = H.new_empty((m, D), dtype=dtype or H.dtype)
    elif dtype is not None and out.dtype != dtype:
        raise TypeError(f"out must be {dtype}, got {out.dtype}")
    po, ldo = _matrix(out, "out", shape=(m, D))
    if out.device != dev:
        raise TypeError(f"out must be on {dev}")
    work = _work(H, lst_scores_workspace(m, d))
    _enqueue("lst_scores", dev, code, _dtype_code(out, "out"), m, D, d, ph, ldh,
             _vector(codes, torch.uint8, "codes", dev),
             _vector(scales, torch.uint8, "scales", dev), po, ldo,
             None if work is None else work.data_ptr())
    return out


@functools.lru_cache(maxsize=256)
def lst_sample_workspace(m: int, D: int) -> int:
    return int(load_library().lst_sample_workspace(m, D))


def lst_sample(logits, u, *, temperature=None, top_k=None, top_p=None, min_p=None, tokens=None,
               prob=None):
    """(tokens, prob): a token for each row of outputs from the random numbers u (one a row, in
    [0, 1)); temperature, top_k, top_p and min_p are device vectors, one value a row, or None."""
    import torch

    px, ldx = _matrix(logits, "logits")
    code = _dtype_code(logits, "logits")
    (m, D), dev = logits.shape, logits.device
    if tokens is None:
        tokens = logits.new_empty(m, dtype=torch.int32)
    if prob is None:
        prob = logits.new_empty(m, dtype=torch.float32)
    work = _work(logits, lst_sample_workspace(m, D))
    f32 = torch.float32
    if u is None:
        raise TypeError("u must be a device vector of float32")
    _enqueue("lst_sample", dev, code, m, D, px, ldx,
             _vector(temperature, f32, "temperature", dev, m),
             _vector(top_k, torch.int32, "top_k", dev, m), _vector(top_p, f32, "top_p", dev, m),
             _vector(min_p, f32, "min_p", dev, m), _vector(u, f32, "u", dev, m),
             _vector(tokens, torch.int32, "tokens", dev, m), _vector(prob, f32, "prob", dev, m),
             None if work is None else work.data_ptr())
    return tokens, prob


# ------------------------------------------------------------------- classes
class _Layer:
    def __init__(self, handle, D: int, d: int, m_max: int, K_max: int, device):
        self._h = handle
        self.D, self.d = D, d
        self.m_max, self.K_max = m_max, K_max
        self.device = device

    def _alloc_outputs(self, m):
        import torch

        return (torch.empty(m, dtype=torch.float32, device=self.device),
                torch.empty((m, self.d), dtype=torch.float32, device=self.device))

    def materialize_W(self, out=None):
        import torch

        if out is None:
            out = torch.empty((self.D, self.d), dtype=torch.float32, device=self.device)
        lst_materialize_W(self._h, out)
        return out

    def sync(self) -> int:
        return lst_sync(self._h)

    def set_graphs(self, enable: bool = True) -> None:
        lst_set_graphs(self._h, enable)

    def profile(self, enable: bool = True) -> None:
        lst_profile_enable(self._h, enable)

    def profile_read(self):
        return lst_profile_read(self._h)

    def stats(self) -> lst_stats_t:
        return lst_stats(self._h)

    def close(self) -> None:
        if self._h is not None:
            lst_free(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class FactoredOutputLayer(_Layer):
    """W = V U with Q = W^T W and U^{-T} kept up to date (section 3 of the paper)."""

    def __init__(self, V, U=None, *, loss="squared", sph_eps=1e-3, m_max=128, K_max=16,
                 cond_max=0.0, stream=None):
        h = lst_init(V, U, loss=loss, sph_eps=sph_eps, m_max=m_max, K_max=K_max,
                     cond_max=cond_max, stream=stream)
        super().__init__(h, V.shape[0], V.shape[1], m_max, K_max, V.device)

    def step(self, H, Y_idx, Y_val, lr, out: Optional[Tuple] = None):
        loss, grad = out if out is not None else self._alloc_outputs(H.shape[0])
        lst_step(self._h, H, Y_idx, Y_val, lr, loss, grad)
        return loss, grad

    def step_solve(self, H, Y_idx, Y_val, lr, out: Optional[Tuple] = None):
        """The step with U_new^T Z = H solved from scratch (lst_step_solve)."""
        loss, grad = out if out is not None else self._alloc_outputs(H.shape[0])
        lst_step_solve(self._h, H, Y_idx, Y_val, lr, loss, grad)
        return loss, grad

    def get_state(self):
        import torch

        Q, U, Uit = (torch.empty((self.d, self.d), dtype=torch.float32, device=self.device)
                     for _ in range(3))
        lst_get_state(self._h, Q, U, Uit)
        return Q, U, Uit

    def get_V(self):
        import torch

        V = torch.empty((self.D, self.d), dtype=torch.float32, device=self.device)
        lst_get_V(self._h, V)
        return V

    def get_shift(self):
        """(c, s) of the shifted spherical loss: W = V U + 1 c^T, s = W^T 1."""
        import torch

        c, s = (torch.empty(self.d, dtype=torch.float32, device=self.device) for _ in range(2))
        lst_get_shift(self._h, c, s)
        return c, s

    def touched_rows(self):
        return lst_touched_rows(self._h, self.m_max * self.K_max)

    def restore(self):
        lst_restore(self._h)

    def set_split_tasks(self, enable: bool = True) -> None:
        lst_set_split_tasks(self._h, enable)

    def stabilize(self, **kw):
        return lst_stabilize(self._h, **kw)

    def stabilize_noalloc(self, **kw):
        return lst_stabilize_noalloc(self._h, **kw)

    def set_stabilize(self, every: int, **kw) -> None:
        lst_set_stabilize(self._h, every, **kw)


class SparseInputLayer:
    """Section 2.2 input layer: W_in (D_in x d) with K-sparse inputs."""

    def __init__(self, W_in, stream=None):
        import torch

        lib = load_library()
        self.D, self.d = W_in.shape
        self.device = W_in.device
        h = _P()
        _check(lib.lst_input_init(ctypes.byref(h), self.D, self.d,
                                  _ptr(W_in, torch.float32, "W_in"), _stream_handle(stream)),
               "lst_input_init")
        self._h = h

    def forward(self, idx, val, out=None):
        import torch

        m, K = idx.shape
        if out is None:
            out = torch.empty((m, self.d), dtype=torch.float32, device=self.device)
        _check(load_library().lst_input_forward(self._h, m, K, _ptr(idx, torch.int32, "idx"),
                                                _ptr(val, torch.float32, "val"),
                                                _ptr(out, torch.float32, "A")), "lst_input_forward")
        return out

    def update(self, idx, val, grad_A, lr):
        import torch

        m, K = idx.shape
        if tuple(grad_A.shape) != (m, self.d):
            raise ValueError("grad_A must be (m, d)")
        _check(load_library().lst_input_update(self._h, m, K, _ptr(idx, torch.int32, "idx"),
                                               _ptr(val, torch.float32, "val"),
                                               _ptr(grad_A, torch.float32, "grad_A"), float(lr)),
               "lst_input_update")

    def get_W(self):
        import torch

        W = torch.empty((self.D, self.d), dtype=torch.float32, device=self.device)
        _check(load_library().lst_input_get_W(self._h, _ptr(W, torch.float32, "W")),
               "lst_input_get_W")
        return W

    def sync(self) -> int:
        return int(load_library().lst_input_sync(self._h))

    def close(self) -> None:
        if self._h is not None:
            load_library().lst_input_free(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class NaiveOutputLayer(_Layer):
    """Explicit W (the O(D d) per example computation), same library and kernels."""

    def __init__(self, W, *, loss="squared", sph_eps=1e-3, m_max=128, K_max=16, stream=None):
        h = lst_naive_init(W, loss=loss, sph_eps=sph_eps, m_max=m_max, K_max=K_max, stream=stream)
        super().__init__(h, W.shape[0], W.shape[1], m_max, K_max, W.device)

    def step(self, H, Y_idx, Y_val, lr, out: Optional[Tuple] = None):
        loss, grad = out if out is not None else self._alloc_outputs(H.shape[0])
        lst_naive_step(self._h, H, Y_idx, Y_val, lr, loss, grad)
        return loss, grad


class Dropout:
    """Dropout whose mask is drawn from (seed, offset, row, column) and never stored: the
    backward pass takes the offset of its forward pass.  It is called by name: torch's autograd
    does not see either."""

    def __init__(self, p: float, seed: int = 0):
        if not 0.0 <= p <= 1.0:
            raise ValueError("p must be in [0, 1]")
        self.p, self.seed = float(p), _word(seed, "seed")

    def forward(self, x, offset=0, *, residual=None, counter=None, out=None):
        return lst_dropout(x, self.p, self.seed, offset, residual=residual, counter=counter,
                           out=out)

    def backward(self, grad_y, offset=0, *, counter=None, out=None):
        return lst_dropout(grad_y, self.p, self.seed, offset, counter=counter, out=out)


class GatedRecurrence:
    """h_t = f_t h_{t-1} + (1 - f_t) x_t with f = sigmoid(g), over packed sequences.

    The backward pass is called by name: torch's autograd does not see either.  Rows that belong
    to no sequence are not written: in outputs of the call's own they hold what the memory held."""

    def __init__(self, d: int, device="cuda"):
        import torch

        load_library()
        self.d = int(d)
        self._status = torch.zeros(1, dtype=torch.int32, device=device)

    def _width(self, x):
        if x.dim() != 2 or x.shape[1] != self.d:
            raise ValueError(f"rows must have {self.d} columns")

    def forward(self, x, g, offsets=None, h0=None, *, n_seq=None, out=None, h_last=None,
                save=False):
        self._width(x)
        return lst_recur_forward(x, g, offsets, h0, n_seq=n_seq, out=out, h_last=h_last,
                                 save=save, status=self._status)

    def backward(self, x, g, grad_y, saved, offsets=None, h0=None, grad_last=None, *, n_seq=None,
                 out=None):
        self._width(x)
        return lst_recur_backward(x, g, grad_y, saved, offsets, h0, grad_last, n_seq=n_seq,
                                  out=out, status=self._status)

    def step(self, x, g, h, slots=None, *, out=None):
        self._width(x)
        return lst_recur_step(x, g, h, slots, out=out, status=self._status)

    def sync(self) -> int:
        """Wait for the device; returns (and clears) the sticky status code."""
        import torch

        torch.cuda.synchronize(self._status.device)
        code = int(self._status.item())
        if code:
            self._status.zero_()
        return code


class EightBitOutputLayer:
    """The outputs O = H W^T of a trained layer, its weights held in 8 bits: W is any D x d matrix,
    or an output layer, whose materialize_W gives one.

    A row takes 129 bytes for each 128 columns begun: a quarter of float32's at d = 512, as many
    at d = 32.  H is rounded to 8 bits in the same way, in each call."""

    def __init__(self, W):
        W = self._weights(W)
        self.D, self.d = W.shape
        self.codes, self.scales = lst_quantize(W)

    @staticmethod
    def _weights(W):
        if not isinstance(W, _Layer):
            return W
        import torch

        # a layer works on the stream of its own: it must not write before the current stream is
        # done with what was in the new tensor's memory, nor be read before it has written
        out = torch.empty((W.D, W.d), dtype=torch.float32, device=W.device)
        torch.cuda.synchronize(out.device)
        W = W.materialize_W(out)
        torch.cuda.synchronize(out.device)
        return W

    def load(self, W) -> None:
        """Take new weights of the same shape, into the same memory."""
        W = self._weights(W)
        if tuple(W.shape) != (self.D, self.d):
            raise ValueError(f"W must be ({self.D}, {self.d})")
        lst_quantize(W, codes=self.codes, scales=self.scales)

    def scores(self, H, *, dtype=None, out=None):
        if H.dim() != 2 or H.shape[1] != self.d:
            raise ValueError(f"H must have {self.d} columns")
        return lst_scores(H, self.codes, self.scales, dtype=dtype, out=out)

    def sample(self, H, u, **settings):
        """(tokens, prob) chosen from the outputs for H: lst_sample's settings."""
        return lst_sample(self.scores(H, dtype=settings.pop("dtype", None)), u, **settings)
