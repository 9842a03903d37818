"""Binding of include/oob_layer.h: the operators of a transformer layer on torch tensors.

Argument checks, output tensors and workspaces only: every step runs in the HIP kernels of liboob_plan.so.  Work is
enqueued on torch's current stream of the tensors' device; nothing waits.  There is no CPU fallback.  No call builds an
autograd graph: what a call makes requires no gradient, whatever its inputs do; gradients are the *_backward calls' results.
"""
from __future__ import annotations

import contextlib
import ctypes as C

from . import binding

OOB_BF16, OOB_FP16, OOB_FP32 = 0, 1, 2
ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4}
LAYER_SYMBOLS = ["oob_layer_linear", "oob_layer_linear_workspace_size", "oob_layer_linear_backward",
                 "oob_layer_linear_backward_workspace_size", "oob_layer_norm", "oob_layer_norm_backward",
                 "oob_layer_norm_backward_workspace_size", "oob_layer_dropout", "oob_layer_attention",
                 "oob_layer_attention_workspace_size", "oob_layer_attention_backward", "oob_layer_attention_backward_workspace_size"]
MASK64 = (1 << 64) - 1
NORMS = {"none": 0, "layer": 1, "rms": 2}


class oob_linear(C.Structure):
    _fields_ = [("dtype", C.c_int), ("act", C.c_int)] + [(n, C.c_int64) for n in "TNK"] + \
               [(n, C.c_void_p) for n in ("x", "w", "bias", "residual", "y", "z")] + \
               [(n + "_stride", C.c_int64) for n in ("x", "w", "residual", "y", "z")]


class oob_linear_grad(C.Structure):
    _fields_ = [("dtype", C.c_int), ("act", C.c_int)] + [(n, C.c_int64) for n in "TNK"] + \
               [(n, C.c_void_p) for n in ("dy", "x", "w", "z", "dx", "dw", "db")] + \
               [(n + "_stride", C.c_int64) for n in ("dy", "x", "w", "z", "dx", "dw")]


class oob_norm(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("dtype", "pre", "post")] + [(n, C.c_float) for n in ("eps", "alpha", "p")] + \
               [(n, C.c_int64) for n in ("T", "C", "gates")] + [(n, C.c_uint64) for n in ("seed", "offset")] + \
               [(n, C.c_void_p) for n in ("x", "z", "weight", "bias", "post_weight", "post_bias", "gate")] + \
               [(n, C.c_int64) for n in ("x_stride", "z_stride")] + [(n, C.c_void_p) for n in ("xp", "h", "saved")]


class oob_norm_grad(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("dxp", "dh")] + [(n, C.c_int64) for n in ("dxp_stride", "dh_stride")] + \
               [(n, C.c_void_p) for n in ("dx", "dz", "dweight", "dbias", "dpost_weight", "dpost_bias", "dgate")]


class oob_attention(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("dtype", "B", "Sq", "Sk", "H", "G", "D", "causal")] + [(n, C.c_float) for n in ("scale", "cap")] + \
               [(n, C.c_void_p) for n in ("q", "k", "v", "key_begin", "key_end", "slopes", "o", "lse")] + \
               [(n + "_stride", C.c_int64 * 3) for n in "qkvo"]


class oob_attention_grad(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("dout", "dq", "dk", "dv")] + [(n + "_stride", C.c_int64 * 3) for n in ("dout", "dq", "dk", "dv")]


_calls = {}
_lib = torch = None  # both loaded with the first call: the planner's users need not wait for them


def _load():
    global _lib, torch
    if _lib is None:
        import torch

        L = binding.load()
        for name, *structs in (("linear", oob_linear), ("linear_backward", oob_linear_grad), ("norm", oob_norm),
                               ("norm_backward", oob_norm, oob_norm_grad), ("attention", oob_attention),
                               ("attention_backward", oob_attention, oob_attention_grad)):
            call, args = getattr(L, "oob_layer_" + name), [C.POINTER(t) for t in structs]
            size = None
            if name != "norm":  # needs no workspace
                size = getattr(L, f"oob_layer_{name}_workspace_size")
                size.argtypes, size.restype = args[:1] if name == "norm_backward" else args, C.c_size_t
            call.argtypes, call.restype = args + ([C.c_void_p, C.c_size_t] if size else []) + [C.c_void_p], C.c_int
            _calls[name] = size, call
        L.oob_layer_dropout.argtypes = [C.c_int, C.c_void_p, C.c_void_p, C.c_int64, C.c_float, C.c_uint64, C.c_uint64, C.c_void_p]
        L.oob_layer_dropout.restype = C.c_int
        _lib = L
    return _lib


_TYPES = {}


def _dtype(t, wide=False):
    """OOB_* code of a tensor's type; wide: 32 bits too."""
    if not _TYPES:
        _TYPES.update({torch.bfloat16: OOB_BF16, torch.float16: OOB_FP16, torch.float32: OOB_FP32})
    code = _TYPES.get(t.dtype)
    if not (code is not None and (wide or code != OOB_FP32)):
        raise ValueError(f"{t.dtype} is not supported here")
    return code


def _rows(t, cols, like, name):
    """A tensor of the type and device of `like` as rows of `cols` values: itself or a view of it."""
    if not (t.dtype is like.dtype and t.get_device() == like.get_device()):
        raise ValueError(f"{name}: type and device have to be {like.dtype}, {like.device}")
    if not (t.dim() >= 1 and t.shape[-1] == cols):
        raise ValueError(f"{name}: the last axis has {t.shape[-1] if t.dim() else 0} values, not {cols}")
    if t.dim() != 2:
        t = t.view(-1, cols)
    if not (t.stride(1) == 1 or cols == 1):
        raise ValueError(f"{name}: the last axis has to be contiguous")
    return t


def _stride(t):
    """Elements between rows (of one row: its length, whatever torch says)."""
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _vector(t, n, like, name):
    if not (t.dtype is like.dtype and t.get_device() == like.get_device() and tuple(t.shape) == (n,) and (n == 1 or t.stride(0) == 1)):
        raise ValueError(f"{name}: a contiguous vector of {n} values of {like.dtype} on {like.device} is wanted")
    return t.data_ptr()


def _stream(at):
    """torch's current stream of device number `at`, as HIP knows it."""
    return torch._C._cuda_getCurrentRawStream(at)


def _enqueue(name, device, *args):
    """Asks for the workspace of a call and enqueues it on the current stream of `device`."""
    at = device.index
    if at is not None and at != torch.cuda.current_device():
        with torch.cuda.device(device):
            return _enqueue(name, torch.device("cuda"), *args)
    size, call = _calls[name]
    refs = [C.byref(a) for a in args]
    stream = _stream(torch.cuda.current_device() if at is None else at)
    if size is None:
        return binding.check(call(*refs, stream), "oob_layer_" + name)
    nbytes = size(*refs[:len(size.argtypes)])
    # the workspace is held until the call is enqueued; torch gives it to later work of this stream only
    ws = torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes else None
    binding.check(call(*refs, ws.data_ptr() if nbytes else None, nbytes, stream), "oob_layer_" + name)


def _act(act):
    code = ACTIVATIONS.get(act)
    if not (code is not None):
        raise ValueError(f"act: one of {', '.join(ACTIVATIONS)}")
    return code


def linear(x, w, bias=None, act="none", residual=None, keep=False):
    """y = act(x w^T + bias) + residual.  x [..., K], w [N, K], bias [N], residual [..., N]: bfloat16 or float16, rows of any
    stride.  keep=True: (y, z) with z = x w^T + bias, which linear_backward wants where there is an activation (z is None without
    one).  No autograd graph is built: gradients are linear_backward's."""
    _load()
    code = _act(act)
    if not (x.is_cuda and w.dim() == 2):
        raise ValueError("x has to be on the GPU and w a matrix")
    N, K = w.shape
    dtype = _dtype(x)
    x2, w2 = _rows(x, K, x, "x"), _rows(w, K, x, "w")
    T = x2.shape[0]
    y = x.new_empty((*x.shape[:-1], N))
    z = torch.empty_like(y) if keep and code else None
    r = None
    if residual is not None:
        if not (residual.shape == y.shape):
            raise ValueError("residual: the result's shape is wanted")
        r = _rows(residual, N, x, "residual")
    args = oob_linear(dtype, code, T, N, K, x2.data_ptr(), w2.data_ptr(), None if bias is None else _vector(bias, N, x, "bias"),
                      None if r is None else r.data_ptr(), y.data_ptr(), None if z is None else z.data_ptr(),
                      _stride(x2), _stride(w2), 0 if r is None else _stride(r), N, N)
    _enqueue("linear", x.device, args)
    return (y, z) if keep else y


def linear_backward(dy, x, w, z=None, act="none", need=("x", "w", "b")):
    """(dx, dw, db) of linear: dz = dy act'(z), dx = dz w, dw = dz^T x, db = sum of dz; None for what `need` does not name.  The
    residual's gradient is dy."""
    _load()
    code = _act(act)
    if not (x.is_cuda and w.dim() == 2):
        raise ValueError("x has to be on the GPU and w a matrix")
    if not (code == 0 or z is not None):
        raise ValueError("z: the backward pass of an activation wants it (linear with keep=True)")
    if not (set(need) <= {"x", "w", "b"}):
        raise ValueError("need: out of x, w, b")
    N, K = w.shape
    dtype = _dtype(x)
    dy2, x2, w2 = _rows(dy, N, x, "dy"), _rows(x, K, x, "x"), _rows(w, K, x, "w")
    T = x2.shape[0]
    if not (dy2.shape[0] == T):
        raise ValueError("dy and x: different numbers of rows")
    z2 = None
    if code:
        z2 = _rows(z, N, x, "z")
        if not (z2.shape[0] == T):
            raise ValueError("z and x: different numbers of rows")
    new = x.new_empty
    dx = new(x.shape) if "x" in need else None
    dw = new((N, K)) if "w" in need else None
    db = new(N) if "b" in need else None
    ptr = lambda t: None if t is None else t.data_ptr()  # noqa: E731
    args = oob_linear_grad(dtype, code, T, N, K, dy2.data_ptr(), x2.data_ptr(), w2.data_ptr(), ptr(z2), ptr(dx), ptr(dw), ptr(db),
                           _stride(dy2), _stride(x2), _stride(w2), 0 if z2 is None else _stride(z2), K, K)
    _enqueue("linear_backward", x.device, args)
    return dx, dw, db


def _norm_args(x, z, xp, h, saved, weight, bias, pre, post, post_weight, post_bias, gate, alpha, eps, p, seed, offset):
    if not (x.is_cuda and x.dim() >= 1):
        raise ValueError("x has to be on the GPU")
    width = x.shape[-1]
    dtype = _dtype(x, wide=True)
    if not (pre in ("layer", "rms") and post in NORMS):
        raise ValueError("pre: layer or rms, post: none, layer or rms")
    if not (0 <= p < 1 and p * 65536 + 0.5 < 65536):
        raise ValueError("p: at least 0 and below 1")
    x2 = _rows(x, width, x, "x")
    T = x2.shape[0]
    z2 = None
    if z is not None:
        if not (z.shape == x.shape):
            raise ValueError("z and x: different shapes")
        z2 = _rows(z, width, x, "z")
    else:
        if not (post == "none" and gate is None and p == 0 and alpha == 1):
            raise ValueError("without z there is nothing to norm, gate, drop or scale")
    if not (post != "none" or (post_weight is None and post_bias is None)):
        raise ValueError("post_weight and post_bias belong to a norm behind the block")
    gates, g = 0, None
    if gate is not None:
        if not (gate.shape[-1] == width and gate.numel() > 0):
            raise ValueError("gate: the last axis is not x's")
        gates = gate.numel() // width
        if not (T > 0 and T % gates == 0):
            raise ValueError(f"gate: {T} rows do not divide among {gates}")
        if not (gate.dtype == x.dtype and gate.device == x.device and gate.is_contiguous()):
            raise ValueError("gate: contiguous, of x's type and device")
        g = gate.data_ptr()
    vec = lambda t, name: None if t is None else _vector(t, width, x, name)  # noqa: E731
    ptr = lambda t: None if t is None else t.data_ptr()  # noqa: E731
    return oob_norm(dtype, NORMS[pre], NORMS[post], eps, alpha, p, T, width, gates, seed & MASK64, offset & MASK64, x2.data_ptr(), ptr(z2),
                    vec(weight, "weight"), vec(bias, "bias"), vec(post_weight, "post_weight"), vec(post_bias, "post_bias"), g,
                    _stride(x2), 0 if z2 is None else _stride(z2), ptr(xp), ptr(h), ptr(saved))


def residual_norm(x, z=None, weight=None, bias=None, pre="layer", post="none", post_weight=None, post_bias=None, gate=None,
                  alpha=1.0, eps=1e-5, p=0.0, seed=0, offset=0):
    """The norms around a block: xp = alpha x + gate * dropout(post(z)), h = pre(xp); (xp, h, saved).

    x: the residual stream [..., C]; z: the block's output, or None (xp is x: the first norm of a model); pre: "layer" or "rms" with
    weight and bias [C]; post: "none" or a norm with post_weight and post_bias; gate [C] or [G, C]: one for each G-th of the rows;
    dropout: dropout(post(z), p, seed, offset), element by element of the rows.  bfloat16, float16 or float32.  saved: statistics
    that the backward pass wants.  No autograd graph is built: gradients are residual_norm_backward's."""
    _load()
    h, xp = x.new_empty(x.shape), x if z is None else x.new_empty(x.shape)
    width = x.shape[-1] if x.dim() else 0
    saved = torch.empty((2 if post == "none" else 4, x.numel() // max(width, 1)), dtype=torch.float32, device=x.device)
    args = _norm_args(x, z, None if z is None else xp, h, saved, weight, bias, pre, post, post_weight, post_bias, gate, alpha, eps, p, seed, offset)
    _enqueue("norm", x.device, args)
    return xp, h, saved


def residual_norm_backward(dxp, dh, xp, z, saved, weight=None, bias=None, pre="layer", post="none", post_weight=None, post_bias=None,
                           gate=None, alpha=1.0, eps=1e-5, p=0.0, seed=0, offset=0):
    """Gradients of residual_norm from those of its results (dxp None: zero), as a dict: "x", "z" and the name of every weight that is
    given (None for the others).  Everything behind `saved` as in the forward call."""
    _load()
    args = _norm_args(xp, z, None, None, saved, weight, bias, pre, post, post_weight, post_bias, gate, alpha, eps, p, seed, offset)
    T, width = args.T, args.C
    if not (saved.dtype == torch.float32 and saved.device == xp.device and saved.is_contiguous() and tuple(saved.shape) == (2 if post == "none" else 4, T)):
        raise ValueError("saved: not that of such a call")
    if not (dh.shape == xp.shape and (dxp is None or dxp.shape == xp.shape)):
        raise ValueError("dxp, dh and xp: different shapes")
    dh2 = _rows(dh, width, xp, "dh")
    dxp2 = None if dxp is None else _rows(dxp, width, xp, "dxp")
    new = lambda t: None if t is None else xp.new_empty(t.shape)  # noqa: E731
    out = {"x": new(xp), "z": new(z), "weight": new(weight), "bias": new(bias), "post_weight": new(post_weight),
           "post_bias": new(post_bias), "gate": new(gate)}
    ptr = lambda t: None if t is None else t.data_ptr()  # noqa: E731
    grad = oob_norm_grad(ptr(dxp2), dh2.data_ptr(), 0 if dxp2 is None else _stride(dxp2), _stride(dh2), *(ptr(t) for t in out.values()))
    _enqueue("norm_backward", xp.device, args, grad)
    return out


def dropout(x, p, seed, offset=0, out=None):
    """keep / (1 - p) * x for a contiguous tensor of any shape (bfloat16, float16, float32); out may be x.  The mask comes from
    (seed, offset + element) alone and is never stored: the backward pass is the same call on the gradient (no autograd
    graph is built)."""
    _load()
    if not (x.is_cuda and x.is_contiguous()):
        raise ValueError("x has to be contiguous and on the GPU")
    dtype = _dtype(x, wide=True)
    if not (0 <= p < 1 and p * 65536 + 0.5 < 65536):
        raise ValueError("p: at least 0 and below 1")
    if out is None:
        out = torch.empty_like(x)
    if not (out.shape == x.shape and out.dtype == x.dtype and out.device == x.device and out.is_contiguous()):
        raise ValueError("out: not like x")
    with contextlib.nullcontext() if x.device.index in (None, torch.cuda.current_device()) else torch.cuda.device(x.device):
        binding.check(_lib.oob_layer_dropout(dtype, x.data_ptr(), out.data_ptr(), x.numel(), p, seed & MASK64, offset & MASK64,
                                             _stream(x.get_device())), "oob_layer_dropout")
    return out


def _heads(t, name, like, B, S, N, D):
    if not (t.dim() == 4 and tuple(t.shape) == (B, S, N, D)):
        raise ValueError(f"{name}: [{B}, {S}, {N}, {D}] is wanted, not {list(t.shape)}")
    if not (t.dtype is like.dtype and t.get_device() == like.get_device()):
        raise ValueError(f"{name}: type and device have to be {like.dtype}, {like.device}")
    if not (D == 1 or t.stride(3) == 1):
        raise ValueError(f"{name}: the last axis has to be contiguous")
    return t.data_ptr(), (C.c_int64 * 3)(*t.stride()[:3])


def _attention_args(q, k, v, o, lse, scale, causal, key_begin, key_end, slopes, cap):
    if not (q.is_cuda and q.dim() == 4 and k.dim() == 4):
        raise ValueError("q and k have to be on the GPU: [batch, length, heads, width]")
    B, Sq, H, D = q.shape
    Sk, G = k.shape[1], k.shape[2]
    if not (1 <= D <= 128):
        raise ValueError("heads of 1 to 128 values are supported")
    if not (G >= 1 and H >= 1 and H % G == 0):
        raise ValueError(f"{H} heads do not divide among {G}")
    dtype = _dtype(q)
    scale = D ** -0.5 if scale is None else scale
    if not (0 < scale < float("inf") and 0 <= cap < float("inf")):
        raise ValueError("scale has to be above 0, cap 0 (none) or above")
    (pq, sq), (pk, sk), (pv, sv) = _heads(q, "q", q, B, Sq, H, D), _heads(k, "k", q, B, Sk, G, D), _heads(v, "v", q, B, Sk, G, D)
    po, so = _heads(o, "o", q, B, Sq, H, D)
    ranges = []
    for t, name in ((key_begin, "key_begin"), (key_end, "key_end")):
        if not (t is None or (t.dtype == torch.int32 and t.device == q.device and tuple(t.shape) == (B, Sq) and t.is_contiguous())):
            raise ValueError(f"{name}: a contiguous int32 [{B}, {Sq}] on {q.device} is wanted")
        ranges.append(None if t is None else t.data_ptr())
    if not (slopes is None or (slopes.dtype == torch.float32 and slopes.device == q.device and tuple(slopes.shape) == (H,) and slopes.is_contiguous())):
        raise ValueError(f"slopes: {H} contiguous float32 values on {q.device} are wanted")
    return oob_attention(dtype, B, Sq, Sk, H, G, D, bool(causal), scale, cap, pq, pk, pv, *ranges,
                         None if slopes is None else slopes.data_ptr(), po, lse.data_ptr(), sq, sk, sv, so)


def attention(q, k, v, scale=None, causal=False, key_begin=None, key_end=None, slopes=None, cap=0.0):
    """(o, lse) with o_i = sum_j softmax_j(s_ij) v_j, s_ij = cap tanh(scale q_i.k_j / cap) - slope |i + Sk - Sq - j| over the keys
    key_begin_i <= j < key_end_i (causal: and j <= i + Sk - Sq).

    q [B, Sq, H, D], k, v [B, Sk, G, D] of any strides with a contiguous last axis, H a multiple of G; bfloat16 or float16, D up to
    128.  scale: D ** -0.5 where None.  key_begin, key_end: int32 [B, Sq] or None; document, prefix and window masks are such ranges
    (document_ranges, prefix_ranges).  slopes: float32 [H] or None; cap 0: none.  A query that sees no key gets 0 and lse -inf,
    whatever it holds; keys that no query of a 128-row tile sees (between those that it does, too) may hold anything, others have to be
    finite.  lse [B, H, Sq] in float32 goes to attention_backward: no autograd graph is built."""
    _load()
    if not (q.dim() == 4):
        raise ValueError("q: [batch, length, heads, width]")
    B, Sq, H, D = q.shape
    o = q.new_empty((B, Sq, H, D))
    lse = torch.empty((B, H, Sq), dtype=torch.float32, device=q.device)
    _enqueue("attention", q.device, _attention_args(q, k, v, o, lse, scale, causal, key_begin, key_end, slopes, cap))
    return o, lse


def attention_backward(do, q, k, v, o, lse, scale=None, causal=False, key_begin=None, key_end=None, slopes=None, cap=0.0, out=None):
    """(dq, dk, dv) of attention from `do`, the gradient of o.  out: three tensors to write them to, of any strides but 0 with a
    contiguous last axis (the parts of one tensor, say)."""
    _load()
    args = _attention_args(q, k, v, o, lse, scale, causal, key_begin, key_end, slopes, cap)
    B, Sq, H, D = q.shape
    Sk, G = k.shape[1], k.shape[2]
    if not (tuple(lse.shape) == (B, H, Sq) and lse.dtype == torch.float32 and lse.device == q.device and lse.is_contiguous()):
        raise ValueError("lse: not that of such a call")
    if out is None:
        out = tuple(t.new_empty(t.shape) for t in (q, k, v))
    parts = [_heads(do, "do", q, B, Sq, H, D), _heads(out[0], "dq", q, B, Sq, H, D), _heads(out[1], "dk", q, B, Sk, G, D),
             _heads(out[2], "dv", q, B, Sk, G, D)]
    grad = oob_attention_grad(*(p for p, _ in parts), *(s for _, s in parts))
    _enqueue("attention_backward", q.device, args, grad)
    return tuple(out)


def document_ranges(lengths, S, device="cuda"):
    """(key_begin, key_end) of documents packed one behind the other into sequences of S tokens, causal within each: `lengths` has a
    list of lengths per sequence.  Tokens behind the last document see nothing and are seen by none."""
    _load()
    begin, end = torch.zeros((len(lengths), S), dtype=torch.int32), torch.zeros((len(lengths), S), dtype=torch.int32)
    for b, docs in enumerate(lengths):
        if not (all(n >= 0 for n in docs) and sum(docs) <= S):
            raise ValueError(f"sequence {b}: documents of {sum(docs)} tokens in {S}")
        at = 0
        for n in docs:
            begin[b, at: at + n] = at
            end[b, at: at + n] = torch.arange(at + 1, at + n + 1, dtype=torch.int32)
            at += n
    return begin.to(device), end.to(device)


def prefix_ranges(lengths, S, device="cuda"):
    """(key_begin, key_end) of sequences whose first lengths[b] tokens are seen by all and whose others are causal."""
    _load()
    prefix = torch.tensor([int(n) for n in lengths], dtype=torch.int32)[:, None]
    if not (bool(((prefix >= 0) & (prefix <= S)).all())):
        raise ValueError("a prefix is longer than the sequence")
    end = torch.maximum(torch.arange(1, S + 1, dtype=torch.int32)[None], prefix)
    return torch.zeros_like(end).to(device), end.to(device)
