"""What the operators' C entries refuse before they look at memory, and the
sizes they ask for, without a GPU."""

import ctypes
import math

import pytest

import ops_tiles as tiles
import paper_2609_25442_amd as wb

F32, BF16, F8 = 0, 1, 2


class Matrix(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("dtype", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("ld", ctypes.c_int64)]


class Args(ctypes.Structure):
    _fields_ = [(f, Matrix) for f in ("x", "x_scales", "weight", "weight_scales", "bias", "residual", "out", "out_scales")]
    _fields_ += [("offsets", ctypes.c_void_p), ("tokens", ctypes.c_void_p), ("num_experts", ctypes.c_int32),
                 ("activation", ctypes.c_int32), ("gated", ctypes.c_int32), ("reserved", ctypes.c_int32)]


def m(rows, cols, dtype=BF16, ld=None, data=4096):
    return Matrix(data, dtype, 0, rows, cols, cols if ld is None else ld)


def linear(**more):
    a = Args()
    a.x, a.weight, a.out = m(4, 64), m(32, 64), m(4, 32)
    for k, v in more.items():
        setattr(a, k, v)
    return a


def workspace(a):
    n = ctypes.c_size_t(0)
    return wb.lib.wb_linear_workspace(ctypes.byref(a), ctypes.byref(n)), n.value


def test_linear_workspace_of_plain_results_is_none():
    assert workspace(linear()) == (wb.WB_OK, 0)
    assert workspace(linear(out=m(4, 32, F32))) == (wb.WB_OK, 0)
    assert workspace(linear(x=m(0, 64), out=m(0, 32))) == (wb.WB_OK, 0)


def test_linear_workspace_of_fp8_results_holds_fp32_rows():
    a = linear(weight=m(4096, 64), out=m(4, 4096, F8), out_scales=m(4, 32, F32))
    rc, n = workspace(a)
    assert rc == wb.WB_OK and n in (0, 4 * 4096 * 4)


def test_linear_workspace_of_long_rows_off_the_grid_holds_copies():
    assert workspace(linear(x=m(2, 7543), weight=m(1337, 7543), out=m(2, 1337))) == (wb.WB_OK, 1339 * 7544 * 2)
    # only what is off the grid
    assert workspace(linear(x=m(24, 6016, data=4106), weight=m(96, 6016), out=m(24, 96))) == (wb.WB_OK, 24 * 6016 * 2)
    assert workspace(linear(x=m(24, 6016), weight=m(96, 6016, ld=6017), out=m(24, 96))) == (wb.WB_OK, 96 * 6016 * 2)
    # with the fp32 rows behind them
    rc, n = workspace(linear(x=m(8, 6001), weight=m(96, 6001), out=m(8, 96, F8), out_scales=m(8, 1, F32)))
    assert rc == wb.WB_OK and n == 104 * 6008 * 2 + 8 * 96 * 4


@pytest.mark.parametrize("more,code", [
    (dict(x=m(4, 63)), wb.WB_EINVAL), (dict(out=m(4, 31)), wb.WB_EINVAL), (dict(out=m(3, 32)), wb.WB_EINVAL),
    (dict(x=m(4, 64, ld=63)), wb.WB_EINVAL), (dict(gated=1), wb.WB_EINVAL), (dict(activation=3), wb.WB_EINVAL),
    (dict(x=m(4, 64, F32)), wb.WB_EUNSUPPORTED), (dict(x=m(4, 64, F8)), wb.WB_EUNSUPPORTED),
    (dict(x=m(4, 64, F8), weight=m(32, 64, F8)), wb.WB_EINVAL),
    (dict(x=m(4, 64, F8), weight=m(32, 64, F8), x_scales=m(4, 1, F32), weight_scales=m(2, 1, F32)), wb.WB_EINVAL),
    (dict(x_scales=m(4, 1, F32)), wb.WB_EINVAL), (dict(bias=m(1, 31, F32)), wb.WB_EINVAL),
    (dict(bias=m(1, 32, F8)), wb.WB_EINVAL), (dict(residual=m(4, 31)), wb.WB_EINVAL),
    (dict(out=m(4, 32, F8)), wb.WB_EINVAL), (dict(out_scales=m(4, 1, F32)), wb.WB_EINVAL),
    (dict(out=m(4, 32, F8), out_scales=m(4, 2, F32)), wb.WB_EINVAL), (dict(offsets=4096), wb.WB_EINVAL),
    (dict(tokens=4096), wb.WB_EINVAL), (dict(num_experts=2), wb.WB_EINVAL), (dict(num_experts=-1), wb.WB_EINVAL),
    (dict(num_experts=3, offsets=4096), wb.WB_EINVAL), (dict(x=m(1 << 22, 64), out=m(1 << 22, 32)), wb.WB_EUNSUPPORTED),
    (dict(x=m(-1, 64)), wb.WB_EINVAL), (dict(x=m(4, 0), weight=m(32, 0)), wb.WB_EINVAL),
])
def test_linear_refuses(more, code):
    a = linear(**more)
    assert workspace(a)[0] == code
    assert wb.lib.wb_last_error()
    assert wb.lib.wb_linear(ctypes.byref(a), None, ctypes.c_size_t(0), None) == code


@pytest.mark.parametrize("more", [
    # extents whose bytes wrap around 64 bits to a few, or to none
    dict(x=m((1 << 21) + 1, 64, ld=1 << 40), out=m((1 << 21) + 1, 32)),
    dict(out=m((1 << 21) + 1, 32, ld=1 << 40), x=m((1 << 21) + 1, 64)),
    dict(weight=m(1 << 23, 64, ld=1 << 40), out=m(4, 1 << 23)),
    dict(weight=m(1 << 41, 64, ld=1 << 40), num_experts=1 << 15, offsets=4096, out=m(4, 1 << 26)),
])
def test_linear_refuses_extents_past_64_bits(more):
    a = linear(**more)
    assert workspace(a)[0] == wb.WB_EINVAL
    assert b"out of range" in wb.lib.wb_last_error()


def test_linear_refuses_memory_the_gpu_cannot_address():
    buf = ctypes.create_string_buffer(1 << 16)
    at = (ctypes.addressof(buf) + 255) // 256 * 256
    a = linear(x=m(4, 64, data=at), weight=m(32, 64, data=at + 8192), out=m(4, 32, data=at + 16384))
    assert wb.lib.wb_linear(ctypes.byref(a), None, ctypes.c_size_t(0), None) == wb.WB_EINVAL


def test_null_arguments_are_refused():
    f, z = wb.lib, ctypes.c_size_t(0)
    assert f.wb_linear(None, None, z, None) == wb.WB_EINVAL
    assert f.wb_linear_workspace(None, ctypes.byref(z)) == wb.WB_EINVAL
    assert f.wb_linear_workspace(ctypes.byref(linear()), None) == wb.WB_EINVAL
    assert f.wb_route(None, None, 1, 0, None, None, z, None) == wb.WB_EINVAL
    assert f.wb_route_backward(None, None, 1, 0, None, None, None, None, None) == wb.WB_EINVAL
    assert f.wb_add_rms_norm(None, None, None, ctypes.c_float(0), None, None, None, None) == wb.WB_EINVAL
    assert f.wb_combine(None, None, None, 1, None, None, None, None, None) == wb.WB_EINVAL
    assert f.wb_route_workspace(ctypes.c_int64(4), 8, None) == wb.WB_EINVAL


@pytest.mark.parametrize("rows,experts,code", [(0, 1, 0), (1, 8, 0), (64, 1024, 0), (65, 256, 0), (4194303, 8, 0),
                                               (-1, 8, wb.WB_EINVAL), (4, 0, wb.WB_EINVAL), (4, 1025, wb.WB_EUNSUPPORTED),
                                               (4194304, 8, wb.WB_EUNSUPPORTED)])
def test_route_workspace(rows, experts, code):
    n = ctypes.c_size_t(0)
    assert wb.lib.wb_route_workspace(ctypes.c_int64(rows), experts, ctypes.byref(n)) == code
    if code == 0:
        # one sum and one count per expert, and the rows sent, for at most 256 blocks of rows
        assert 8 * experts + 4 <= n.value <= 256 * (8 * experts + 4)


def test_operators_refuse_cpu_tensors():
    import torch

    if torch.cuda.is_available():
        pytest.skip("the GPU's own refusals are tested there")
    x = torch.zeros(2, 8)
    with pytest.raises(wb.WbError):
        wb.add_rms_norm(x, x[0], out_dtype="f16")
    with pytest.raises(wb.WbError):
        wb.linear(x, x, activation="tanh")
    with pytest.raises(wb.WbError):
        wb.expert_linear(x, x, None)


def test_linear_takes_tiles_that_one_launch_can():
    """128 x 128 tiles would be expected to end first, but are 8.7 million; of 256 x 256 there are 2.2 million, and
    their 128 columns hold the scales of a gated result, so that no fp32 rows are asked for."""
    rows, n = 4194303, 34000
    a = linear(x=m(rows, 64), weight=m(n, 64), out=m(rows, n // 2, F8), out_scales=m(rows, 133, F32), gated=1)
    assert workspace(a) == (wb.WB_OK, 0)


def test_linear_refuses_more_tiles_than_a_launch_takes():
    """Before anything is launched, and with every size within its own limit."""
    rows, n = 4194303, 1 << 26
    for k in (64, 63):  # rows on the 16-byte grid, and rows that would be copied onto it first
        a = linear(x=m(rows, k), weight=m(n, k), out=m(rows, n))
        assert workspace(a)[0] == wb.WB_EUNSUPPORTED
        assert b"tiles" in wb.lib.wb_last_error()


def product(rows, n, k, f8, gated=False, experts=0, residual=False, out="bf16", x_rows=None):
    """The C call's arguments of contiguous operands."""
    t, cols, xr = F8 if f8 else BF16, n // 2 if gated else n, rows if x_rows is None else x_rows
    nb = lambda c: -(-c // 128)  # noqa: E731
    a = Args()
    a.x, a.weight, a.gated = m(xr, k, t), m(n * max(1, experts), k, t), int(gated)
    if f8:
        a.x_scales, a.weight_scales = m(xr, nb(k), F32), m(nb(n) * max(1, experts), nb(k), F32)
    if experts:
        a.num_experts, a.offsets = experts, 4096
        a.tokens = 4096 if x_rows is not None else None
    if residual:
        a.residual = m(rows, cols)
    a.out = m(rows, cols, {"bf16": BF16, "f32": F32, "f8e4m3": F8}[out])
    if out == "f8e4m3":
        a.out_scales = m(rows, nb(cols), F32)
    return a


def test_workspaces_are_those_of_the_tiles_the_rule_takes():
    """The copies of the operands and the fp32 rows of fp8 results depend on the tile: the rule written out in
    ops_tiles gives the library's bytes exactly."""
    import random

    rng = random.Random(3)
    size = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    seen = set()
    for _ in range(4000):
        rows, n, k = size(1, 16384), 2 * size(8, 8192), size(16, 8192)
        if rng.random() < 0.6:
            rows, n, k = (max(1, rows // 64 * 64), max(64, n // 64 * 64), max(16, k // 16 * 16))
        more = dict(gated=rng.random() < 0.5, residual=rng.random() < 0.3, out=rng.choice(["bf16", "f32", "f8e4m3", "f8e4m3"]),
                    experts=rng.choice([0, 0, 1, 8, 40]))
        if more["experts"] and rng.random() < 0.5:
            more["x_rows"] = max(1, rows // 4)
        f8 = rng.random() < 0.5
        tile, way, need = tiles.form(rows, n, k, f8, **more)
        assert workspace(product(rows, n, k, f8, **more)) == (wb.WB_OK, need), (rows, n, k, f8, more, tile, way)
        seen.add((tile, way))
    assert len(seen) > 20


def test_linear_workspace_of_fp8_results_is_the_tile_s():
    # 16 x 32 tiles hold no scale's columns; 128 x 128 do, and 256 x 256 those of a gated result
    assert workspace(product(4, 4096, 4096, False, out="f8e4m3")) == (wb.WB_OK, 4 * 4096 * 4)
    assert workspace(product(4, 4096, 64, False, out="f8e4m3")) == (wb.WB_OK, 0)  # one step: 128 x 128 ends before two launches
    assert workspace(product(1024, 8192, 1024, True, out="f8e4m3")) == (wb.WB_OK, 0)
    assert workspace(product(8192, 8192, 1024, False, gated=True, out="f8e4m3")) == (wb.WB_OK, 0)
    assert workspace(product(128, 4096, 7168, True, gated=True, experts=32, x_rows=32, out="f8e4m3")) == (wb.WB_OK, 128 * 2048 * 4)


def test_sizes_of_the_products_tests_take_every_tile():
    """Each tile in each type and way that the table has, plain and stacked, plain and gated."""
    want = {(t, f8, "direct") for t in range(len(tiles.TABLE)) for f8 in (False, True)}
    want |= {(t, f8, "registers") for t, c in enumerate(tiles.TABLE) for f8 in (False, True) if c["by_registers"][f8]}
    assert set(tiles.SIZES) == want
    for (tile, f8, way), sizes in tiles.SIZES.items():
        for s in sizes:
            assert tiles.form_of_size(f8, s)[:2] == (tile, way), (tile, f8, way, s)
        assert {bool(s[4]) for s in sizes} == {False, True}, (tile, f8, way)
        assert {tiles.FORMS[s[0]].get("gated", False) for s in sizes} == {False, True}, (tile, f8, way)
