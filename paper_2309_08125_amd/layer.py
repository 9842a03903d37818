"""Binding of include/oob_layer.h: the operators of a transformer layer on torch tensors.

Argument checks, output tensors and workspaces only: every step runs in the HIP kernels of liboob_plan.so.  Work is
enqueued on torch's current stream of the tensors' device; nothing waits.  There is no CPU fallback.
"""
from __future__ import annotations

import ctypes as C

from . import binding

OOB_BF16, OOB_FP16, OOB_FP32 = 0, 1, 2
ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4}
LAYER_SYMBOLS = ["oob_layer_linear", "oob_layer_linear_workspace_size", "oob_layer_linear_backward",
                 "oob_layer_linear_backward_workspace_size"]


class oob_linear(C.Structure):
    _fields_ = [("dtype", C.c_int), ("act", C.c_int)] + [(n, C.c_int64) for n in "TNK"] + \
               [(n, C.c_void_p) for n in ("x", "w", "bias", "residual", "y", "z")] + \
               [(n + "_stride", C.c_int64) for n in ("x", "w", "residual", "y", "z")]


class oob_linear_grad(C.Structure):
    _fields_ = [("dtype", C.c_int), ("act", C.c_int)] + [(n, C.c_int64) for n in "TNK"] + \
               [(n, C.c_void_p) for n in ("dy", "x", "w", "z", "dx", "dw", "db")] + \
               [(n + "_stride", C.c_int64) for n in ("dy", "x", "w", "z", "dx", "dw")]


_lib = None


def _load():
    global _lib
    if _lib is None:
        L = binding.load()
        for name, struct in (("linear", oob_linear), ("linear_backward", oob_linear_grad)):
            size, call = getattr(L, f"oob_layer_{name}_workspace_size"), getattr(L, f"oob_layer_{name}")
            size.argtypes, size.restype = [C.POINTER(struct)], C.c_size_t
            call.argtypes, call.restype = [C.POINTER(struct), C.c_void_p, C.c_size_t, C.c_void_p], C.c_int
        _lib = L
    return _lib


def _need(ok, what):
    if not ok:
        raise ValueError(what)


def _codes(types):
    import torch

    return {getattr(torch, n): c for n, c in types}


_TYPES = {}


def _dtype(t, wide=False):
    """OOB_* code of a tensor's type; wide: 32 bits too."""
    if not _TYPES:
        _TYPES.update(_codes((("bfloat16", OOB_BF16), ("float16", OOB_FP16), ("float32", OOB_FP32))))
    code = _TYPES.get(t.dtype)
    _need(code is not None and (wide or code != OOB_FP32), f"{t.dtype} is not supported here")
    return code


def _rows(t, cols, like, name):
    """A tensor of the type and device of `like` as rows of `cols` values: itself or a view of it."""
    _need(t.dtype == like.dtype and t.device == like.device, f"{name}: type and device have to be {like.dtype}, {like.device}")
    _need(t.dim() >= 1 and t.shape[-1] == cols, f"{name}: the last axis has {t.shape[-1] if t.dim() else 0} values, not {cols}")
    if t.dim() != 2:
        t = t.view(-1, cols)
    _need(t.stride(1) == 1 or cols == 1, f"{name}: the last axis has to be contiguous")
    return t


def _stride(t):
    """Elements between rows (of one row: its length, whatever torch says)."""
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _vector(t, n, like, name):
    _need(t.dtype == like.dtype and t.device == like.device and tuple(t.shape) == (n,) and (n == 1 or t.stride(0) == 1),
          f"{name}: a contiguous vector of {n} values of {like.dtype} on {like.device} is wanted")
    return t.data_ptr()


def _run(name, args, device):
    """Asks for the workspace of a call and enqueues it on the current stream of `device`."""
    import torch

    lib = _load()
    if device.index is not None and device.index != torch.cuda.current_device():
        with torch.cuda.device(device):
            return _run(name, args, torch.device("cuda"))
    ref = C.byref(args)
    nbytes = getattr(lib, f"oob_layer_{name}_workspace_size")(ref)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=device).data_ptr() if nbytes else None
    binding.check(getattr(lib, f"oob_layer_{name}")(ref, ws, nbytes, torch.cuda.current_stream().cuda_stream), f"oob_layer_{name}")


def _act(act):
    code = ACTIVATIONS.get(act)
    _need(code is not None, f"act: one of {', '.join(ACTIVATIONS)}")
    return code


def linear(x, w, bias=None, act="none", residual=None, keep=False):
    """y = act(x w^T + bias) + residual.  x [..., K], w [N, K], bias [N], residual [..., N]: bfloat16 or float16, rows of any
    stride.  keep=True: (y, z) with z = x w^T + bias, which linear_backward wants where there is an activation (z is None without
    one)."""
    import torch

    code = _act(act)
    _need(x.is_cuda and w.dim() == 2, "x has to be on the GPU and w a matrix")
    N, K = w.shape
    dtype = _dtype(x)
    x2, w2 = _rows(x, K, x, "x"), _rows(w, K, x, "w")
    T = x2.shape[0]
    y = torch.empty((*x.shape[:-1], N), dtype=x.dtype, device=x.device)
    z = torch.empty_like(y) if keep and code else None
    r = None
    if residual is not None:
        _need(residual.shape == y.shape, "residual: the result's shape is wanted")
        r = _rows(residual, N, x, "residual")
    args = oob_linear(dtype, code, T, N, K, x2.data_ptr(), w2.data_ptr(), None if bias is None else _vector(bias, N, x, "bias"),
                      None if r is None else r.data_ptr(), y.data_ptr(), None if z is None else z.data_ptr(),
                      _stride(x2), _stride(w2), 0 if r is None else _stride(r), N, N)
    _run("linear", args, x.device)
    return (y, z) if keep else y


def linear_backward(dy, x, w, z=None, act="none", need=("x", "w", "b")):
    """(dx, dw, db) of linear: dz = dy act'(z), dx = dz w, dw = dz^T x, db = sum of dz; None for what `need` does not name.  The
    residual's gradient is dy."""
    import torch

    code = _act(act)
    _need(x.is_cuda and w.dim() == 2, "x has to be on the GPU and w a matrix")
    _need(code == 0 or z is not None, "z: the backward pass of an activation wants it (linear with keep=True)")
    _need(set(need) <= {"x", "w", "b"}, "need: out of x, w, b")
    N, K = w.shape
    dtype = _dtype(x)
    dy2, x2, w2 = _rows(dy, N, x, "dy"), _rows(x, K, x, "x"), _rows(w, K, x, "w")
    T = x2.shape[0]
    _need(dy2.shape[0] == T, "dy and x: different numbers of rows")
    z2 = None
    if code:
        z2 = _rows(z, N, x, "z")
        _need(z2.shape[0] == T, "z and x: different numbers of rows")
    new = lambda *shape: torch.empty(shape, dtype=x.dtype, device=x.device)  # noqa: E731
    dx = new(*x.shape) if "x" in need else None
    dw = new(N, K) if "w" in need else None
    db = new(N) if "b" in need else None
    ptr = lambda t: None if t is None else t.data_ptr()  # noqa: E731
    args = oob_linear_grad(dtype, code, T, N, K, dy2.data_ptr(), x2.data_ptr(), w2.data_ptr(), ptr(z2), ptr(dx), ptr(dw), ptr(db),
                           _stride(dy2), _stride(x2), _stride(w2), 0 if z2 is None else _stride(z2), K, K)
    _run("linear_backward", args, x.device)
    return dx, dw, db
