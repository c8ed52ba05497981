"""What the trainer's operators' C entries refuse before they look at memory,
the workspaces that they ask for, and what the binding refuses without a GPU."""

import ctypes

import pytest

import paper_2609_25442_amd as wb
from test_ops_cpu import BF16, F8, F32, Matrix, m


class Tokens(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("bytes", ctypes.c_int32), ("reserved", ctypes.c_int32), ("count", ctypes.c_int64)]


P = ctypes.c_void_p(4096)
I64, F = ctypes.c_int64, ctypes.c_float
MANY = 4194304  # one row more than there may be


def ref(v):
    return None if v is None else ctypes.byref(v) if isinstance(v, (Matrix, Tokens)) else v


def call(name, *args):
    return getattr(wb.lib, name)(*[ref(a) for a in args])


def ids(count=4, nbytes=8, data=4096):
    return Tokens(data, nbytes, 0, count)


def embedding(t=None, w=None, out=None, first=0):
    return call("wb_embedding", t or ids(), w or m(9, 64), F(1), I64(first), out or m(4, 64), None)


def embedding_backward(t=None, d=None, dw=None, first=0, ws=P, n=1 << 40):
    return call("wb_embedding_backward", t or ids(), d or m(4, 64), F(1), I64(first), dw or m(9, 64), ws, ctypes.c_size_t(n), None)


def norm(x=None, r=None, w=None, b=None, eps=1e-5, total=None, out=None, mean=P, inv=P):
    return call("wb_add_layer_norm", x or m(4, 64), r, w or m(1, 64), b, F(eps), total, out or m(4, 64), mean, inv, None)


def norm_backward(d=None, t=None, w=None, dt=None, mean=P, inv=P, dx=None, dr=None, dw=None, db=None, n=1 << 40):
    return call("wb_add_layer_norm_backward", d or m(4, 64), t or m(4, 64), w or m(1, 64), dt, mean, inv, dx or m(4, 64), dr, dw, db,
                P, ctypes.c_size_t(n), None)


def dispatch(x=None, positions=P, tokens=P, k=2, first=None, last=None, out=None, name="wb_dispatch"):
    a, b = x or m(4, 64), out or m(8, 64)
    if name == "wb_dispatch_backward":
        a, b = b, a
    return call(name, a, positions, tokens, k, first, last, b, None)


def collect_backward(d=None, y=m(8, 64), positions=P, tokens=P, gates=P, k=2, first=None, last=None, dy=m(8, 64), dg=P):
    return call("wb_combine_backward", d or m(4, 64), y, positions, tokens, gates, k, first, last, dy, dg, None)


def activate(x=None, act=1, gated=0, out=None, codes=None, scales=None):
    return call("wb_activate", x or m(4, 64), act, gated, out or m(4, 64), codes, scales, None)


def activate_backward(d=None, x=None, scales=None, act=1, gated=0, dx=None):
    return call("wb_activate_backward", d or m(4, 64), x or m(4, 64), scales, act, gated, dx or m(4, 64), None)


E, U = wb.WB_EINVAL, wb.WB_EUNSUPPORTED


@pytest.mark.parametrize("f,more,code", [
    (embedding, dict(t=ids(nbytes=2)), E), (embedding, dict(t=ids(-1)), E), (embedding, dict(t=ids(MANY)), U),
    (embedding, dict(w=m(MANY, 64)), U), (embedding, dict(w=m(9, 64, F8)), E), (embedding, dict(w=m(9, 64, ld=63)), E),
    (embedding, dict(out=m(4, 63)), E), (embedding, dict(out=m(3, 64)), E), (embedding, dict(out=m(4, 64, F8)), E),
    (embedding, dict(first=-1), E), (embedding, dict(first=(1 << 62) + 1), E), (embedding, dict(w=m(9, 0), out=m(4, 0)), E),
    (embedding, dict(t=ids(data=None)), E), (embedding, dict(t=ids(data=4100)), E), (embedding, dict(w=m(-1, 64)), E),
    (embedding_backward, dict(d=m(3, 64)), E), (embedding_backward, dict(d=m(4, 64, F8)), E), (embedding_backward, dict(dw=m(9, 65)), E),
    (embedding_backward, dict(dw=m(MANY, 64)), U), (embedding_backward, dict(first=-1), E),
    (norm, dict(x=m(4, 64, F8)), E), (norm, dict(w=m(1, 63)), E), (norm, dict(w=m(2, 64)), E), (norm, dict(b=m(1, 63)), E),
    (norm, dict(b=m(1, 64, F8)), E), (norm, dict(eps=-1.0), E), (norm, dict(eps=float("nan")), E), (norm, dict(r=m(4, 64)), E),
    (norm, dict(total=m(4, 64)), E), (norm, dict(r=m(4, 64), total=m(4, 63)), E), (norm, dict(r=m(3, 64), total=m(4, 64)), E),
    (norm, dict(out=m(4, 64, F8)), E), (norm, dict(inv=None), E), (norm, dict(mean=ctypes.c_void_p(4098)), E),
    (norm, dict(x=m(MANY, 64), out=m(MANY, 64)), U), (norm, dict(x=m(4, 1 << 27), out=m(4, 1 << 27)), E),
    (norm_backward, dict(d=m(3, 64)), E), (norm_backward, dict(dt=m(4, 63)), E), (norm_backward, dict(dx=m(4, 64, F8)), E),
    (norm_backward, dict(dr=m(4, 65)), E), (norm_backward, dict(dw=m(1, 63)), E), (norm_backward, dict(db=m(1, 64)), E),
    (norm_backward, dict(dw=m(1, 64), db=m(2, 64)), E), (norm_backward, dict(inv=None), E), (norm_backward, dict(t=m(4, 64, F8)), E),
    (dispatch, dict(k=0), E), (dispatch, dict(k=65), U), (dispatch, dict(first=P), E), (dispatch, dict(last=P), E),
    (dispatch, dict(positions=None), E), (dispatch, dict(tokens=None), E), (dispatch, dict(x=m(4, 63)), E), (dispatch, dict(x=m(4, 64, F8)), E),
    (dispatch, dict(out=m(8, 64, F8)), E), (dispatch, dict(x=m(MANY, 64)), U), (dispatch, dict(out=m(1 << 31, 64)), U),
    (dispatch, dict(positions=ctypes.c_void_p(4098)), E), (dispatch, dict(name="wb_dispatch_backward", x=m(4, 63)), E),
    (dispatch, dict(name="wb_dispatch_backward", k=0), E), (dispatch, dict(name="wb_dispatch_backward", out=m(8, 64, F8)), E),
    (collect_backward, dict(y=None, dg=None, dy=None), E), (collect_backward, dict(y=None), E), (collect_backward, dict(dg=None), E),
    (collect_backward, dict(gates=None), E), (collect_backward, dict(dy=m(7, 64)), E), (collect_backward, dict(y=m(8, 63)), E),
    (collect_backward, dict(y=m(8, 64, F8)), E), (collect_backward, dict(k=65), U), (collect_backward, dict(d=m(4, 64, F8)), E),
    (activate, dict(act=3), E), (activate, dict(act=-1), E), (activate, dict(x=m(4, 63), gated=1), E), (activate, dict(gated=1), E),
    (activate, dict(out=m(4, 64, F8)), E), (activate, dict(x=m(4, 64, F8)), E), (activate, dict(codes=m(4, 64, F8)), E),
    (activate, dict(codes=m(4, 64), scales=m(4, 1, F32)), E), (activate, dict(codes=m(4, 64, F8), scales=m(4, 2, F32)), E),
    (activate, dict(codes=m(4, 63, F8), scales=m(4, 1, F32)), E), (activate, dict(x=m(MANY, 64), out=m(MANY, 64)), U),
    (activate_backward, dict(d=m(4, 63)), E), (activate_backward, dict(x=m(4, 64, F8)), E), (activate_backward, dict(scales=m(4, 1, F32)), E),
    (activate_backward, dict(x=m(4, 64, F8), scales=m(4, 2, F32)), E), (activate_backward, dict(dx=m(4, 63)), E),
    (activate_backward, dict(x=m(4, 64, F8), scales=m(4, 1, BF16)), E), (activate_backward, dict(act=9), E),
    (activate_backward, dict(x=m(4, 128, F8), gated=1, scales=m(4, 1, F32), dx=m(4, 128)), E),
])
def test_refused(f, more, code):
    assert f(**more) == code
    assert wb.lib.wb_last_error()


def test_refused_without_arguments():
    z = ctypes.c_size_t(0)
    assert call("wb_embedding", None, m(1, 1), F(1), I64(0), m(1, 1), None) == E
    assert call("wb_embedding_backward", ids(), None, F(1), I64(0), m(1, 1), P, z, None) == E
    assert call("wb_add_layer_norm", None, None, None, None, F(0), None, None, None, None, None) == E
    assert call("wb_add_layer_norm_backward", None, None, None, None, None, None, None, None, None, None, None, z, None) == E
    assert call("wb_dispatch", None, P, P, 1, None, None, None, None) == E
    assert call("wb_dispatch_backward", None, P, P, 1, None, None, None, None) == E
    assert call("wb_combine_backward", None, None, P, P, P, 1, None, None, None, None, None) == E
    assert call("wb_activate", None, 1, 0, None, None, None, None) == E
    assert call("wb_activate_backward", None, None, None, 1, 0, None, None) == E
    assert call("wb_embedding_backward_workspace", I64(1), I64(1), I64(1), None) == E
    assert call("wb_add_layer_norm_backward_workspace", I64(1), I64(1), None) == E


@pytest.mark.parametrize("f", [embedding, embedding_backward, norm, norm_backward, dispatch, collect_backward, activate, activate_backward])
def test_memory_the_gpu_cannot_address_is_refused(f):
    assert f() == E  # addresses that no allocation has


def size(name, *args):
    n = ctypes.c_size_t(0)
    return call(name, *[I64(a) for a in args], ctypes.byref(n)), n.value


def test_workspaces():
    name = "wb_embedding_backward_workspace"
    assert size(name, 0, 10, 8) == (0, 0)
    # sorted keys and their tokens; past one chunk two fp32 rows for each as well
    rc, n = size(name, 16, 10, 8)
    assert rc == 0 and n == 2 * 64
    for count, rows, cols in ((17, 1, 1), (8192, 128256, 4096), (8193, 128256, 4096), (4194303, 4194303, 64)):
        rc, n = size(name, count, rows, cols)
        assert rc == 0 and n >= 8 * count
        assert n <= 16 * count + (2 << 20) + 4096 + 8 * cols * (count // 16 + 1)
    for bad, code in (((-1, 1, 1), E), ((MANY, 1, 1), U), ((1, -1, 1), E), ((1, MANY, 1), U), ((1, 1, 0), E), ((1, 1, (1 << 26) + 1), E)):
        assert size(name, *bad)[0] == code
    name = "wb_add_layer_norm_backward_workspace"
    for rows, cols in ((0, 8), (1, 1), (16384, 4096), (4194303, 64), (3, 1 << 26)):
        rc, n = size(name, rows, cols)
        assert rc == 0 and 8 * cols * min(rows, 1) <= n <= 8 * max(rows, 1) + 8 * 2048 * max(cols, 2048)
    for bad, code in (((-1, 1), E), ((MANY, 1), U), ((1, 0), E), ((1, (1 << 26) + 1), E)):
        assert size(name, *bad)[0] == code


def test_the_binding_refuses_cpu_tensors_and_names():
    import torch

    if torch.cuda.is_available():
        pytest.skip("the GPU's own refusals are tested there")
    x = torch.zeros(4, 8)
    for f in (lambda: wb.embedding(x, x, out_dtype="f16"), lambda: wb.add_layer_norm(x, x[0], out_dtype="half"),
              lambda: wb.activate(x, "tanh"), lambda: wb.embedding_backward(x, x, 4, out_dtype="i8")):
        with pytest.raises(wb.WbError):
            f()
