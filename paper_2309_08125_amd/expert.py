"""Binding of include/oob_expert.h: the operators of a layer with experts, and clipping at the end of a step, on torch tensors.

As in layer.py: argument checks, output tensors and workspaces only, work on torch's current stream of the tensors' device, no CPU
fallback, no autograd graph: gradients are the *_backward calls' results."""
from __future__ import annotations

import ctypes as C
import math

from . import binding, layer
from .layer import _act, _dtype, _rows, _stride

SCORES = {"softmax": 0, "sigmoid": 1}
EXPERT_SYMBOLS = ["oob_expert_route", "oob_expert_route_backward", "oob_expert_rows", "oob_expert_rows_workspace_size", "oob_expert_linear",
                  "oob_expert_linear_workspace_size", "oob_expert_linear_backward", "oob_expert_linear_backward_workspace_size", "oob_expert_sum",
                  "oob_expert_sum_backward", "oob_clip_norm", "oob_clip_overlap", "oob_clip_scale", "oob_clip_workspace_size"]
MAX_EXPERTS, MAX_CHOICES = 1024, 64


class oob_route(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("dtype", "score", "renormalize", "E", "k", "groups", "keep_groups", "group_best")] + \
               [("scale", C.c_float), ("T", C.c_int64), ("logits", C.c_void_p), ("logits_stride", C.c_int64)] + \
               [(n, C.c_void_p) for n in ("bias", "experts", "weights")]


class oob_expert_linear_t(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("dtype", "act", "E", "per")] + [(n, C.c_int64) for n in "RTNK"] + \
               [(n, C.c_void_p) for n in ("offsets", "rows", "x", "w", "bias", "y", "z")] + \
               [(n + "_stride", C.c_int64) for n in ("x", "w", "expert", "y", "z")]


class oob_expert_linear_grad(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("dy", "dx", "dw", "db")] + [(n + "_stride", C.c_int64) for n in ("dy", "dx")]


class oob_expert_sum_t(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("dtype", "k")] + [(n, C.c_int64) for n in "TRC"] + \
               [(n, C.c_void_p) for n in ("y", "place", "weights", "residual", "out")] + [(n + "_stride", C.c_int64) for n in ("y", "residual", "out")]


_calls = {}
_lib = torch = None


def _load():
    global _lib, torch
    if _lib is None:
        layer._load()
        import torch

        L, p, i, n = binding.load(), C.c_void_p, C.c_int, C.c_int64
        route, linear, grad, total = (C.POINTER(t) for t in (oob_route, oob_expert_linear_t, oob_expert_linear_grad, oob_expert_sum_t))
        for name, args in (("oob_expert_route", [route, p]), ("oob_expert_route_backward", [route, p, p, n, p]),
                           ("oob_expert_rows", [p, n, i, i, p, p, p, p, C.c_size_t, p]),
                           ("oob_expert_linear", [linear, p, C.c_size_t, p]), ("oob_expert_linear_backward", [linear, grad, p, C.c_size_t, p]),
                           ("oob_expert_sum", [total, p]), ("oob_expert_sum_backward", [total, p, n, p, n, p, p]),
                           ("oob_clip_overlap", [i, p, p, p, p, p]), ("oob_clip_norm", [i, p, p, p, p, p, C.c_size_t, p]),
                           ("oob_clip_scale", [i, p, p, p, p, C.c_float, p, p, p, C.c_size_t, p])):
            call = _calls[name] = getattr(L, name)
            call.argtypes, call.restype = args, C.c_int
        for name, args in (("oob_expert_rows", [n, i]), ("oob_expert_linear", [linear]), ("oob_expert_linear_backward", [linear, grad]),
                           ("oob_clip", [i, p])):
            size = _calls[name + "_workspace_size"] = getattr(L, name + "_workspace_size")
            size.argtypes, size.restype = args, C.c_size_t
        _lib = L
    return _lib


def _ptr(t):
    return None if t is None else t.data_ptr()


def _enqueue(name, at, *args, size=None, out=None, read=()):
    """Enqueues a call on the current stream of GPU number `at`, with a workspace where it takes one (size: what that goes by); out: the
    caller's tensor that the call writes to and refuses where it shares memory with those that it reads."""
    if at != torch._C._cuda_getDevice():
        with torch.cuda.device(at):
            return _enqueue(name, at, *args, size=size, out=out, read=read)
    stream = layer._stream(at)
    if size is None:
        rc = _calls[name](*args, stream)
    else:
        nbytes = _calls[size[0]](*size[1:])
        # the workspace is held until the call is enqueued; torch gives it to later work of this stream only
        ws = torch.empty(nbytes, dtype=torch.uint8, device="cuda") if nbytes else None
        rc = _calls[name](*args, ws.data_ptr() if nbytes else None, nbytes, stream)
    if rc:
        if out is not None and not all([_apart(out, m) for t in read if t is not None for m in (t if t.dim() == 3 else (t,))]):
            raise ValueError("out: it shares memory with what the call reads")
        binding.check(rc, name)


def _part(t):
    """Where a tensor lies: first byte, end, and of rows (all but its last axis) their pitch and length in bytes."""
    size, at, n = t.element_size(), t.data_ptr(), t.shape
    span = sum((c - 1) * s for c, s in zip(n, t.stride())) + 1 if t.numel() else 0
    return at, at + span * size, t.stride(0) * size if t.dim() == 2 and n[0] > 1 else 0, n[-1] * size


def _apart(a, b):
    """Whether two tensors share no memory; columns of one matrix of rows do not."""
    a0, a1, pitch, wide = _part(a)
    b0, b1, other, long = _part(b)
    if a1 <= b0 or b1 <= a0:
        return True
    gap = (b0 - a0) % pitch if pitch and pitch == other else 0
    return gap >= wide and gap + long <= pitch


def _numbers(t, shape, like, name):
    """A contiguous int32 tensor on the device of `like`."""
    if not (t.dtype is torch.int32 and t.get_device() == like.get_device() and t.shape == shape and t.is_contiguous()):
        raise ValueError(f"{name}: a contiguous int32 {list(shape)} on {like.device} is wanted")
    return t.data_ptr()


def _floats(t, shape, like, name):
    if not (t.dtype is torch.float32 and t.get_device() == like.get_device() and t.shape == shape and t.is_contiguous()):
        raise ValueError(f"{name}: contiguous float32 {list(shape)} on {like.device} is wanted")
    return t.data_ptr()


def _route_args(logits, k, score, renormalize, scale):
    if not (logits.is_cuda and logits.dim() >= 1):
        raise ValueError("logits have to be on the GPU")
    E = logits.shape[-1]
    if not (1 <= E <= MAX_EXPERTS and 1 <= k <= min(E, MAX_CHOICES)):
        raise ValueError(f"1 to {MAX_EXPERTS} experts and at most {MAX_CHOICES} choices of them are supported, not {k} of {E}")
    if score not in SCORES:
        raise ValueError(f"score: one of {', '.join(SCORES)}")
    if not math.isfinite(scale):
        raise ValueError("scale has to be finite")
    dtype = _dtype(logits, wide=True)
    rows = _rows(logits, E, logits, "logits")
    return oob_route(dtype, SCORES[score], bool(renormalize), E, k, 1, 1, 1, scale, rows.shape[0], rows.data_ptr(), _stride(rows), None, None, None)


def route(logits, k, score="softmax", bias=None, groups=1, keep_groups=None, group_best=2, renormalize=True, scale=1.0):
    """(experts, weights) of every token: the k experts with the largest score + bias, of equals the first, and scale times their
    scores (renormalize: their share of the k scores' sum).

    logits [..., E] in bfloat16, float16 or float32, rows of any stride that do not overlap or one for all (stride 0), E up to 1024; score: "softmax" or "sigmoid"; bias: float32 [E]
    or None, counts for the choice alone.  groups > 1: the experts are so many runs of neighbours, and only the keep_groups (all where None)
    take part whose group_best (1 or 2) largest add up to most.  An expert whose logit is -inf comes after all others and has score 0; a
    token that has no other gets weights 0.  experts int32 [..., k] in falling order, weights float32 [..., k].  No autograd graph
    is built: gradients are route_backward's."""
    _load()
    args = _route_args(logits, k, score, renormalize, scale)
    keep_groups = groups if keep_groups is None else keep_groups
    if not (1 <= groups <= 64 and args.E % groups == 0 and 1 <= keep_groups <= groups and group_best in (1, 2)):
        raise ValueError(f"groups: 1 to 64 that divide {args.E} experts, keep_groups at most as many, group_best 1 or 2")
    if not (k <= keep_groups * (args.E // groups)):
        raise ValueError(f"{keep_groups} groups of {args.E // groups} experts do not hold {k}")
    args.groups, args.keep_groups, args.group_best = groups, keep_groups, group_best
    if bias is not None:
        args.bias = _floats(bias, (args.E,), logits, "bias")
    shape = (*logits.shape[:-1], k)
    new = logits.new_empty
    experts, weights = new(shape, dtype=torch.int32), new(shape, dtype=torch.float32)
    args.experts, args.weights = experts.data_ptr(), weights.data_ptr()
    _enqueue("oob_expert_route", logits.get_device(), C.byref(args))
    return experts, weights


def route_backward(dweights, logits, experts, score="softmax", renormalize=True, scale=1.0):
    """The logits' gradient of route from that of its weights; experts: those of the forward call (its bias and groups have no part)."""
    _load()
    args = _route_args(logits, experts.shape[-1], score, renormalize, scale)
    shape = (*logits.shape[:-1], args.k)
    args.experts = _numbers(experts, shape, logits, "experts")
    d = _floats(dweights, shape, logits, "dweights")
    out = logits.new_empty(logits.shape)
    _enqueue("oob_expert_route_backward", logits.get_device(), C.byref(args), d, out.data_ptr(), args.E)
    return out


def expert_rows(experts, E, first=0):
    """(offsets, rows, place) that put the chosen pairs in order of their experts first .. first + E - 1; pairs of others (-1, say)
    are left out.

    experts int32 [..., k], contiguous.  offsets int32 [E + 1]: rows offsets[e] .. offsets[e + 1] - 1 are those of expert first + e;
    rows int32 [pairs]: the pair (its number in `experts`) of each row, pairs of one expert in their own order, -1 behind the last row; place, like
    experts: the row of each pair, -1 for those left out."""
    _load()
    if not (experts.is_cuda and experts.dtype == torch.int32 and experts.is_contiguous()):
        raise ValueError("experts: contiguous int32 on the GPU are wanted")
    if not (1 <= E <= MAX_EXPERTS and -1 << 31 <= first < 1 << 31):
        raise ValueError(f"1 to {MAX_EXPERTS} experts are supported")
    n, new = experts.numel(), experts.new_empty
    offsets, rows, place = new(E + 1), new(n), new(experts.shape)
    at = experts.get_device()
    if at != torch._C._cuda_getDevice():
        with torch.cuda.device(at):
            _enqueue_rows(experts, n, first, E, offsets, rows, place, at)
    else:
        _enqueue_rows(experts, n, first, E, offsets, rows, place, at)
    return offsets, rows, place


def _enqueue_rows(experts, n, first, E, offsets, rows, place, at):
    nbytes = _lib.oob_expert_rows_workspace_size(n, E)
    ws = torch.empty(nbytes, dtype=torch.uint8, device="cuda") if nbytes else None
    rc = _lib.oob_expert_rows(experts.data_ptr(), n, first, E, offsets.data_ptr(), rows.data_ptr(), place.data_ptr(), ws.data_ptr() if nbytes else None,
                              nbytes, layer._stream(at))
    if rc:
        binding.check(rc, "oob_expert_rows")


def _linear_args(x, w, offsets, rows, act):
    if not (x.is_cuda and w.dim() == 3):
        raise ValueError("x has to be on the GPU and w [experts, N, K]")
    E, N, K = w.shape
    if not (1 <= E <= MAX_EXPERTS and N >= 1 and K >= 1):
        raise ValueError(f"1 to {MAX_EXPERTS} experts are supported, and no empty matrix")
    dtype = _dtype(x)
    x2 = _rows(x, K, x, "x")
    if not (w.dtype is x.dtype and w.get_device() == x.get_device() and (K == 1 or w.stride(2) == 1)):
        raise ValueError(f"w: {x.dtype} on {x.device} is wanted, the last axis contiguous")
    T, per, R = x2.shape[0], 1, x2.shape[0]
    if rows is not None:
        R = rows.numel()
        if not (R == 0 if T == 0 else R % T == 0 and R > 0):
            raise ValueError(f"rows: {R} pairs do not divide among {T} tokens")
        per = R // T if T else 1
        rows = _numbers(rows, rows.shape, x, "rows")
    args = oob_expert_linear_t(dtype, _act(act), E, per, R, T, N, K, _numbers(offsets, (E + 1,), x, "offsets"), rows, x2.data_ptr(),
                               w.data_ptr(), None, None, None)
    args.x_stride = _stride(x2)
    args.w_stride = w.stride(1) if N > 1 else K
    args.expert_stride = w.stride(0) if E > 1 else N * K
    return args


def expert_linear(x, w, offsets, bias=None, rows=None, act="none", keep=False, out=None):
    """Row r of expert e, offsets[e] <= r < offsets[e + 1]: y[r] = act(x[token] w[e]^T + bias[e]).

    x [T, K] with rows [R] of expert_rows: row r is that of token rows[r] // (R // T); or x [R, K], in order already (rows None).  w [E, N,
    K], bias [E, N]; bfloat16 or float16, rows of any stride that do not overlap, of x also one for all (stride 0).  y [R, N], or `out`, which shares no memory with what is read; rows that are no expert's stay as they are (in a
    new y: whatever memory held).  keep=True: (y, z) with z = x w^T + bias, which the backward pass wants where there is an
    activation (z is None without one).  No autograd graph is built: gradients are expert_linear_backward's."""
    _load()
    args = _linear_args(x, w, offsets, rows, act)
    y = x.new_empty((args.R, args.N)) if out is None else _out(out, args.R, args.N, x, "out")
    z = x.new_empty((args.R, args.N)) if keep and args.act else None
    if bias is not None:
        if not (bias.dtype is x.dtype and bias.get_device() == x.get_device() and bias.shape == (args.E, args.N) and bias.is_contiguous()):
            raise ValueError(f"bias: a contiguous [{args.E}, {args.N}] of {x.dtype} on {x.device} is wanted")
        args.bias = bias.data_ptr()
    args.y, args.y_stride, args.z, args.z_stride = y.data_ptr(), _stride(y), _ptr(z), args.N
    ref = C.byref(args)
    _enqueue("oob_expert_linear", x.get_device(), ref, size=("oob_expert_linear_workspace_size", ref), out=out, read=(x, w, bias, offsets, rows))
    return (y, z) if keep else y


def _out(t, R, cols, like, name):
    """A matrix to write to; no two of its rows may share memory."""
    if not (t.dim() == 2 and t.shape[0] == R):
        raise ValueError(f"{name}: [{R}, {cols}] is wanted")
    t = _rows(t, cols, like, name)
    if not (R <= 1 or t.stride(0) >= cols):
        raise ValueError(f"{name}: its rows overlap")
    return t


def expert_linear_backward(dy, x, w, offsets, z=None, rows=None, act="none", need=("x", "w", "b"), out=None):
    """(dx, dw, db) of expert_linear: dz = dy act'(z), dx[r] = dz[r] w[e] (a row each: expert_sum(dx, place) adds those of a token),
    dw[e] = sum of dz[r]^T x[token], db[e] = sum of dz[r], 0 for an expert without rows; None for what `need` does not name.  out: where
    dx goes, no memory that the call reads; rows that are no expert's stay as they are."""
    _load()
    args = _linear_args(x, w, offsets, rows, act)
    if not (args.act == 0 or z is not None):
        raise ValueError("z: the backward pass of an activation wants it (expert_linear with keep=True)")
    if not (set(need) <= {"x", "w", "b"}):
        raise ValueError("need: out of x, w, b")
    if not (out is None or "x" in need):
        raise ValueError("out: dx is not among what is needed")
    dy2 = _rows(dy, args.N, x, "dy")
    if not (dy2.shape[0] == args.R):
        raise ValueError(f"dy: {args.R} rows are wanted")
    if args.act:
        z2 = _rows(z, args.N, x, "z")
        if not (z2.shape[0] == args.R):
            raise ValueError(f"z: {args.R} rows are wanted")
        args.z, args.z_stride = z2.data_ptr(), _stride(z2)
    dx = None
    if "x" in need:
        dx = x.new_empty((args.R, args.K)) if out is None else _out(out, args.R, args.K, x, "out")
    dw = x.new_empty((args.E, args.N, args.K)) if "w" in need else None
    db = x.new_empty((args.E, args.N)) if "b" in need else None
    grad = oob_expert_linear_grad(dy2.data_ptr(), _ptr(dx), _ptr(dw), _ptr(db), _stride(dy2), args.K if dx is None else _stride(dx))
    refs = C.byref(args), C.byref(grad)
    _enqueue("oob_expert_linear_backward", x.get_device(), *refs, size=("oob_expert_linear_backward_workspace_size", *refs), out=out,
             read=(dy2, x, w, z, offsets, rows))
    return dx, dw, db


def _sum_args(y, place, weights):
    if not (y.is_cuda and y.dim() == 2 and place.dim() >= 1 and y.shape[1] >= 1):
        raise ValueError("y has to be on the GPU, [rows, columns], and place [..., choices]")
    k = place.shape[-1]
    if not (1 <= k <= MAX_CHOICES):
        raise ValueError(f"1 to {MAX_CHOICES} choices are supported")
    dtype = _dtype(y, wide=True)
    y = _rows(y, y.shape[1], y, "y")
    return oob_expert_sum_t(dtype, k, place.numel() // k, y.shape[0], y.shape[1], y.data_ptr(), _numbers(place, place.shape, y, "place"),
                            None if weights is None else _floats(weights, place.shape, y, "weights"), None, None, _stride(y), 0, 0)


def expert_sum(y, place, weights=None, residual=None):
    """out[t] = residual[t] + sum over j of weights[t, j] y[place[t, j]], in the order of j.

    y [R, C] in bfloat16, float16 or float32, rows of any stride that do not overlap or one for all (stride 0), those of the residual too; place int32 [..., k] of expert_rows (what is out of 0 .. R-1 has no part);
    weights float32 like place, or None: 1; residual [..., C] or None.  The result is [..., C].  No autograd graph is built: gradients are
    expert_sum_backward's."""
    _load()
    args = _sum_args(y, place, weights)
    out = y.new_empty((*place.shape[:-1], args.C))
    if residual is not None:
        if not (residual.shape == out.shape):
            raise ValueError("residual: the result's shape is wanted")
        r = _rows(residual, args.C, y, "residual")
        args.residual, args.residual_stride = r.data_ptr(), _stride(r)
    args.out, args.out_stride = out.data_ptr(), args.C
    _enqueue("oob_expert_sum", y.get_device(), C.byref(args))
    return out


def expert_sum_backward(dout, y, place, weights=None, need=("y", "weights"), out=None):
    """(dy, dweights) of expert_sum: dy[place[t, j]] = weights[t, j] dout[t], dweights[t, j] = dout[t] . y[place[t, j]] (0 where the
    place is out of range); None for what `need` does not name.  out: where dy goes, no memory that the call reads; rows that are nobody's stay as they are.  No two
    places may be the same (expert_rows makes such).  The residual's gradient is dout."""
    _load()
    args = _sum_args(y, place, weights)
    if not (set(need) <= {"y", "weights"} and need):
        raise ValueError("need: out of y, weights")
    if not (out is None or "y" in need):
        raise ValueError("out: dy is not among what is needed")
    if not (dout.shape == (*place.shape[:-1], args.C)):
        raise ValueError("dout: the result's shape is wanted")
    d = _rows(dout, args.C, y, "dout")
    dy = None
    if "y" in need:
        dy = y.new_empty((args.R, args.C)) if out is None else _out(out, args.R, args.C, y, "out")
    dweights = y.new_empty(place.shape, dtype=torch.float32) if "weights" in need else None
    _enqueue("oob_expert_sum_backward", y.get_device(), C.byref(args), d.data_ptr(), _stride(d), _ptr(dy), args.C if dy is None else _stride(dy),
             _ptr(dweights), out=out, read=(y, d, place, weights))
    return dy, dweights


def _tensors(tensors, name):
    """Host arrays of the tensors' addresses, sizes and types, and their GPU."""
    n = len(tensors)
    if not n:
        raise ValueError(f"{name}: no tensors")
    at = tensors[0].get_device()
    _dtype(tensors[0], wide=True)  # fills the table of types
    codes = layer._TYPES
    types = [codes.get(t.dtype, -1) for t in tensors]
    if at < 0 or min(types) < 0 or not all([t.is_contiguous() and t.get_device() == at for t in tensors]):
        raise ValueError(f"{name}: contiguous tensors of bfloat16, float16 or float32 on one GPU are wanted")
    return n, at, (C.c_void_p * n)(*[t.data_ptr() for t in tensors]), [t.numel() for t in tensors], types


def gradient_norm(tensors):
    """The root of the sum of all squares of contiguous tensors (bfloat16, float16, float32, mixed) as a float32 scalar on their
    device; squares are summed in 64 bits, and a norm that passes 32 bits is an infinity."""
    _load()
    tensors = list(tensors)
    n, at, ptrs, sizes, types = _tensors(tensors, "tensors")
    sizes, types = (C.c_int64 * n)(*sizes), (C.c_int * n)(*types)
    norm = tensors[0].new_empty((), dtype=torch.float32)
    _enqueue("oob_clip_norm", at, n, ptrs, sizes, types, norm.data_ptr(), size=("oob_clip_workspace_size", n, sizes))
    return norm


def clip_gradients(tensors, max_norm, norm=None, out=None):
    """Scales contiguous tensors by max_norm / norm where their norm is above max_norm and finite, and leaves them as they are otherwise;
    returns the norm.

    norm: a float32 scalar on the tensors' device to go by in place of gradient_norm(tensors), one that all ranks have added up, say.
    out: as many tensors of the same sizes and types for the results; without it they are changed in place.  What is written may share no memory
    with anything else that is written or read."""
    _load()
    tensors = list(tensors)
    n, at, ptrs, sizes, types = _tensors(tensors, "tensors")
    max_norm = float(max_norm)
    if not (max_norm >= 0):
        raise ValueError("max_norm: at least 0")
    to = ptrs
    if out is not None:
        m, of, to, out_sizes, out_types = _tensors(list(out), "out")
        if not (m == n and of == at and out_sizes == sizes and out_types == types):
            raise ValueError("out: not like the tensors")
    sizes, types = (C.c_int64 * n)(*sizes), (C.c_int * n)(*types)
    given = None
    if norm is not None:
        given = _floats(norm, norm.shape, tensors[0], "norm")
        if norm.numel() != 1:
            raise ValueError("norm: one value is wanted")
    if _lib.oob_clip_overlap(n, ptrs, to, sizes, types, given):
        raise ValueError("tensors that are written share memory with one another or with what is read")
    if given:
        size = ("oob_clip_workspace_size", 0, sizes)
    else:
        norm = tensors[0].new_empty((), dtype=torch.float32)
        size = ("oob_clip_workspace_size", n, sizes)
    _enqueue("oob_clip_scale", at, n, ptrs, to, sizes, types, max_norm, given, None if given else norm.data_ptr(), size=size)
    return norm
