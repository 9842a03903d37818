"""Host logic of the operators of a transformer layer that needs no GPU: exported symbols, refusals, workspace sizes."""
import ctypes as C
import os
import re

import pytest

import paper_2309_08125_amd as P
from paper_2309_08125_amd import layer as L

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x10000  # never dereferenced: every call below fails its host-side checks or has nothing to do


def lib():
    return L._load()


def test_library_exports_every_declared_symbol():
    text = open(os.path.join(ROOT, "paper_2309_08125_amd", "include", "oob_layer.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = sorted(set(re.findall(r"\b(oob_layer_\w+)\s*\(", text)))
    assert names == sorted(P.LAYER_SYMBOLS) and all(hasattr(lib(), n) for n in names)


def make(struct, **kw):
    s = struct()
    for k, v in kw.items():
        setattr(s, k, v)
    return s


LINEAR = dict(dtype=0, act=0, T=4, N=16, K=8, x=FAKE, w=FAKE, y=FAKE, x_stride=8, w_stride=8, y_stride=16)


@pytest.mark.parametrize("bad", [dict(dtype=2), dict(dtype=-1), dict(act=5), dict(act=-1), dict(T=-1), dict(N=0), dict(K=0), dict(T=1 << 31),
                                 dict(x=0), dict(w=0), dict(y=0), dict(x=FAKE + 1), dict(y=FAKE + 1), dict(x_stride=7), dict(w_stride=7),
                                 dict(y_stride=15), dict(residual=FAKE, residual_stride=15), dict(z=FAKE, z_stride=15), dict(bias=FAKE + 1)])
def test_linear_refuses(bad):
    p = make(L.oob_linear, **{**LINEAR, **bad})
    assert lib().oob_layer_linear(C.byref(p), FAKE, 1 << 40, None) == P.OOB_EINVAL


def test_linear_workspaces():
    assert lib().oob_layer_linear(None, None, 0, None) == P.OOB_EINVAL
    ok = make(L.oob_linear, **LINEAR)
    assert lib().oob_layer_linear(C.byref(ok), FAKE + 8, 1 << 40, None) == P.OOB_EINVAL  # workspace off 256 bytes
    odd = make(L.oob_linear, **{**LINEAR, "K": 7, "x_stride": 7, "w_stride": 7})        # rows that do not start at 16 bytes: packed
    need = lib().oob_layer_linear_workspace_size(C.byref(odd))
    assert need >= (4 + 16) * 8 * 2 and lib().oob_layer_linear(C.byref(odd), FAKE, need - 256, None) == P.OOB_ECAPACITY
    empty = make(L.oob_linear, **{**LINEAR, "T": 0, "x": 0, "y": 0})
    assert lib().oob_layer_linear(C.byref(empty), None, 0, None) == P.OOB_OK
    # the backward pass takes one product after the other: the larger of their needs, behind dz and the bias's sums
    g = make(L.oob_linear_grad, dtype=0, act=3, T=100, N=2061, K=1030, dy=FAKE, x=FAKE, w=FAKE, z=FAKE, dx=FAKE, dw=FAKE, db=FAKE,
             dy_stride=2061, x_stride=1030, w_stride=1030, z_stride=2061, dx_stride=1030, dw_stride=1030)
    both = lib().oob_layer_linear_backward_workspace_size(C.byref(g))
    parts = []
    for out in ("dx", "dw"):
        one = make(L.oob_linear_grad, **{n: getattr(g, n) for n, _ in g._fields_})
        setattr(one, out, None)
        parts.append(lib().oob_layer_linear_backward_workspace_size(C.byref(one)))
    assert both == max(parts) and lib().oob_layer_linear_backward(C.byref(g), FAKE, both - 1, None) == P.OOB_ECAPACITY
    for bad in (dict(z=0), dict(dy=0), dict(w=0), dict(x=0), dict(dx_stride=1029), dict(dw_stride=1029), dict(dy_stride=2060), dict(db=FAKE + 1)):
        b = make(L.oob_linear_grad, **{n: getattr(g, n) for n, _ in g._fields_})
        for k, v in bad.items():
            setattr(b, k, v)
        assert lib().oob_layer_linear_backward(C.byref(b), FAKE, 1 << 40, None) == P.OOB_EINVAL, bad


NORM = dict(dtype=0, pre=1, post=0, eps=1e-5, alpha=1.0, p=0.0, T=6, C=16, gates=0, x=FAKE, z=FAKE, x_stride=16, z_stride=16, xp=FAKE, h=FAKE)


@pytest.mark.parametrize("bad", [dict(dtype=3), dict(pre=0), dict(pre=3), dict(post=3), dict(eps=-1.0), dict(eps=float("nan")), dict(p=1.0),
                                 dict(p=-0.1), dict(p=float("nan")), dict(p=0.999999), dict(T=-1), dict(C=0), dict(C=16385), dict(gates=4, gate=FAKE),
                                 dict(gates=2), dict(gates=-1), dict(x=0), dict(x_stride=15), dict(z_stride=15), dict(xp=0), dict(h=0),
                                 dict(x=FAKE + 1), dict(dtype=2, h=FAKE + 2), dict(z=0, p=0.1), dict(z=0, alpha=0.5), dict(z=0, post=1),
                                 dict(saved=FAKE + 2)])
def test_norm_refuses(bad):
    p = make(L.oob_norm, **{**NORM, **bad})
    assert lib().oob_layer_norm(C.byref(p), None) == P.OOB_EINVAL


def test_norm_backward_refuses():
    p = make(L.oob_norm, **{**NORM, "saved": FAKE})
    grad = dict(dh=FAKE, dh_stride=16, dx=FAKE, dz=FAKE)
    need = lib().oob_layer_norm_backward_workspace_size(C.byref(p))
    assert need > 0
    g = make(L.oob_norm_grad, **grad)
    assert lib().oob_layer_norm_backward(C.byref(p), C.byref(g), FAKE, need - 1, None) == P.OOB_ECAPACITY
    assert lib().oob_layer_norm_backward(C.byref(p), C.byref(g), FAKE + 4, need, None) == P.OOB_EINVAL
    for bad in (dict(dh=0), dict(dx=0), dict(dz=0), dict(dh_stride=15), dict(dxp=FAKE, dxp_stride=15), dict(dweight=FAKE + 1)):
        g = make(L.oob_norm_grad, **{**grad, **bad})
        assert lib().oob_layer_norm_backward(C.byref(p), C.byref(g), FAKE, 1 << 40, None) == P.OOB_EINVAL, bad
    gated = make(L.oob_norm, **{**NORM, "saved": FAKE, "gates": 2, "gate": FAKE})
    g = make(L.oob_norm_grad, **grad)
    assert lib().oob_layer_norm_backward(C.byref(gated), C.byref(g), FAKE, 1 << 40, None) == P.OOB_EINVAL  # no dgate


def test_dropout_refuses():
    call = lambda **k: lib().oob_layer_dropout(k.get("dtype", 0), k.get("x", FAKE), k.get("y", FAKE), k.get("n", 8), k.get("p", 0.1), 1, 0, None)  # noqa: E731
    for bad in (dict(dtype=3), dict(x=0), dict(y=0), dict(n=-1), dict(p=1.0), dict(p=-0.5), dict(p=float("nan")), dict(x=FAKE + 1), dict(dtype=2, y=FAKE + 2)):
        assert call(**bad) == P.OOB_EINVAL, bad
    assert call(n=0, x=0, y=0) == P.OOB_OK


def attention(**kw):
    p = L.oob_attention()
    for k, v in {**dict(dtype=0, B=1, Sq=8, Sk=8, H=4, G=2, D=16, scale=0.25, cap=0.0, q=FAKE, k=FAKE, v=FAKE, o=FAKE, lse=FAKE), **kw}.items():
        if k.endswith("_stride"):
            getattr(p, k)[:] = v
        else:
            setattr(p, k, v)
    for n in "qkvo":
        if n + "_stride" not in kw:
            getattr(p, n + "_stride")[:] = (8 * 64, 64, 16)
    return p


@pytest.mark.parametrize("bad", [dict(dtype=2), dict(B=-1), dict(Sq=-1), dict(Sk=-1), dict(H=0), dict(G=0), dict(G=3), dict(D=0), dict(D=129),
                                 dict(scale=0.0), dict(scale=-1.0), dict(scale=float("inf")), dict(scale=float("nan")), dict(cap=-1.0),
                                 dict(cap=float("nan")), dict(q=0), dict(k=0), dict(v=0), dict(o=0), dict(q=FAKE + 1), dict(key_begin=FAKE + 2),
                                 dict(slopes=FAKE + 2), dict(k_stride=(64, -64, 16)), dict(B=1 << 20, Sq=1 << 20), dict(Sk=1 << 29)])
def test_attention_refuses(bad):
    p = attention(**bad)
    assert lib().oob_layer_attention(C.byref(p), FAKE, 1 << 62, None) == P.OOB_EINVAL


def test_attention_workspaces():
    assert lib().oob_layer_attention_workspace_size(C.byref(attention())) == 0
    odd = attention(D=15)  # heads of no multiple of 8: keys and values are packed
    need = lib().oob_layer_attention_workspace_size(C.byref(odd))
    assert need >= 2 * 8 * 2 * 16 * 2 and lib().oob_layer_attention(C.byref(odd), FAKE, need - 1, None) == P.OOB_ECAPACITY
    assert lib().oob_layer_attention(C.byref(attention(Sq=0)), None, 0, None) == P.OOB_OK
    g = L.oob_attention_grad(FAKE, FAKE, FAKE, FAKE, *[(C.c_int64 * 3)(512, 64, 16) for _ in range(4)])
    need = lib().oob_layer_attention_backward_workspace_size(C.byref(attention()), C.byref(g))
    assert need > 0 and lib().oob_layer_attention_backward(C.byref(attention()), C.byref(g), FAKE, need - 1, None) == P.OOB_ECAPACITY
    g.dq = None
    assert lib().oob_layer_attention_backward(C.byref(attention()), C.byref(g), FAKE, 1 << 40, None) == P.OOB_EINVAL


def test_ranges_of_documents_and_prefixes():
    b, e = P.document_ranges([[2, 0, 3], [6]], 6, device="cpu")
    assert b.tolist() == [[0, 0, 2, 2, 2, 0], [0] * 6] and e.tolist() == [[1, 2, 3, 4, 5, 0], [1, 2, 3, 4, 5, 6]]
    b, e = P.prefix_ranges([0, 3], 4, device="cpu")
    assert b.tolist() == [[0] * 4] * 2 and e.tolist() == [[1, 2, 3, 4], [3, 3, 3, 4]]
    with pytest.raises(ValueError):
        P.document_ranges([[4, 3]], 6, device="cpu")
    with pytest.raises(ValueError):
        P.prefix_ranges([7], 6, device="cpu")
