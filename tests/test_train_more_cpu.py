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
