"""What else the trainer's operators' C entries refuse before they look at memory."""

import ctypes

import pytest

import paper_2609_25442_amd as wb
from test_ops_cpu import BF16, F8, F32, m
from test_train_cpu import E, MANY, P, U, call


def collect(y=None, positions=P, tokens=P, gates=P, k=2, residual=None, first=None, last=None, out=None):
    return call("wb_collect", y or m(8, 64), positions, tokens, gates, k, residual, first, last, out or m(4, 64), None)


@pytest.mark.parametrize("more,code", [
    (dict(k=0), E), (dict(k=65), U), (dict(first=P), E), (dict(last=P), E), (dict(positions=None), E), (dict(tokens=None), E),
    (dict(gates=None), E), (dict(y=m(8, 63)), E), (dict(y=m(8, 64, F8)), E), (dict(y=m(8, 64, ld=63)), E), (dict(y=m(1 << 31, 64)), U),
    (dict(y=m(-1, 64)), E), (dict(out=m(MANY, 64)), U), (dict(out=m(4, 64, F8)), E), (dict(out=m(4, 65)), E), (dict(out=m(-1, 64)), E),
    (dict(residual=m(3, 64)), E), (dict(residual=m(4, 64, F8)), E), (dict(residual=m(4, 65, F32)), E),
    (dict(positions=ctypes.c_void_p(4098)), E), (dict(gates=ctypes.c_void_p(4098)), E), (dict(y=m(8, 64, BF16, data=4097)), E), (dict(), E),
])
def test_collect_refuses(more, code):
    assert collect(**more) == code
    assert wb.lib.wb_last_error()


def test_collect_refuses_without_arguments():
    assert call("wb_collect", None, P, P, P, 1, None, None, None, m(1, 1), None) == E
    assert call("wb_collect", m(1, 1), P, P, P, 1, None, None, None, None, None) == E


@pytest.mark.parametrize("count,rows,cols,code", [
    (8192, 1, 1 << 26, wb.WB_EHIP),        # the joins' launch
    (4194303, 1, 1 << 20, wb.WB_EHIP),     # the sums' one too
    (8192, 4194303, 1 << 22, E), (4194303, 4194303, 8192, E), (16, 9, 1 << 26, E),  # one launch takes these: refused for their memory
])
def test_an_embedding_gradient_past_a_launch_is_refused_before_anything_else(count, rows, cols, code):
    """Before its memory is looked up, and so before its first launch, which would leave d_weight partly written."""
    from test_train_cpu import F, I64, ids

    assert call("wb_embedding_backward", ids(count), m(count, cols), F(1), I64(0), m(rows, cols), P, ctypes.c_size_t(1 << 50), None) == code
    if code == wb.WB_EHIP:
        assert b"embedding gradient" in wb.lib.wb_last_error()
