"""The operators on the GPU against their formulas in 64 bits, at the sizes,
strides, types and masks where a kernel can go wrong. Tolerances follow from
the operations (ops_ref): fp32 sums of so many terms, one rounding to the
output's type."""

import ctypes
import math

import pytest
import torch

import paper_2609_25442_amd as wb
import ops_ref as ref
from gpu_util import say

pytestmark = pytest.mark.gpu
NAMES = {torch.float32: "f32", torch.bfloat16: "bf16"}


def gpu(t):
    return None if t is None else t.cuda()


# ---- norm --------------------------------------------------------------------------------------

NORM_SHAPES = [(1, 1), (1, 7), (3, 8), (5, 127), (4, 128), (2, 129), (3, 512), (7, 513), (5, 1000), (3, 1024), (2, 1025),
               (9, 1500), (3, 2050), (4, 4096), (3, 7168), (2, 16384), (2, 16390), (1, 32768), (2, 40001), (0, 64)]


@pytest.mark.parametrize("out", ["f32", "bf16", "f8e4m3"])
@pytest.mark.parametrize("shape", NORM_SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_norm(shape, out):
    say("norm", shape, out)
    rows, cols = shape
    for seed, (xt, rt, wt) in enumerate([("bf16", "bf16", "bf16"), ("f32", None, "f32"), ("bf16", "f32", "bf16"),
                                         ("f32", "bf16", "f32"), ("bf16", None, "f32")]):
        x = ref.randn(rows, cols, seed=seed, dtype=xt, scale=3.0)
        r = ref.randn(rows, cols, seed=seed + 50, dtype=rt) if rt else None
        w = ref.randn(cols, seed=seed + 100, dtype=wt, scale=0.2) + torch.ones((), dtype=ref.TORCH[wt])
        y, s, total = wb.add_rms_norm(gpu(x), gpu(w), gpu(r), eps=1e-5, out_dtype=out)
        torch.cuda.synchronize()
        want, err, t, terr = ref.norm(x, w, r, 1e-5)
        assert (total is None) == (r is None) and (s is None) == (out != "f8e4m3")
        if r is not None:
            assert total.dtype == r.dtype
            ref.check(total, t, terr, "total")
        if out == "f8e4m3":
            if rows:
                ref.check_f8(y, s, want, err, "norm")
        else:
            assert y.dtype == ref.TORCH[out]
            ref.check(y, want, err, "norm")


@pytest.mark.parametrize("pad,skip", [(0, 1), (3, 0), (5, 3), (8, 8)])
@pytest.mark.parametrize("cols", [5, 264, 1500, 4099])
def test_norm_of_rows_that_start_anywhere(cols, pad, skip):
    say("norm strided", cols, pad, skip)
    x, r = ref.randn(6, cols, seed=1, dtype="bf16"), ref.randn(6, cols, seed=2, dtype="bf16")
    w = ref.randn(cols, seed=3, dtype="bf16")
    for out in ("bf16", "f8e4m3"):
        y, s, total = wb.add_rms_norm(ref.strided(x, pad, skip), gpu(w), ref.strided(r, pad + 1, skip + 1), out_dtype=out)
        y0, s0, total0 = wb.add_rms_norm(gpu(x), gpu(w), gpu(r), out_dtype=out)
        assert torch.equal(y.view(torch.uint8), y0.view(torch.uint8)) and torch.equal(total, total0)
        assert s is None or torch.equal(s, s0)


def test_norm_keeps_nan_and_zero_rows_to_themselves():
    x = ref.randn(6, 700, seed=1, dtype="f32")
    x[1] = 0
    x[2, 5] = math.nan
    x[3, 600] = math.inf
    w = torch.ones(700)
    y, _, _ = wb.add_rms_norm(gpu(x), gpu(w), eps=1e-6)
    want, err, _, _ = ref.norm(x, w, None, 1e-6)
    for t in (0, 1, 4, 5):
        ref.check(y[t:t + 1], want[t:t + 1], err[t:t + 1], f"row {t}")
    assert torch.isnan(y[2]).all() and torch.isnan(y[3, 600]) and torch.all(y[3, :600] == 0)
    q, s, _ = wb.add_rms_norm(gpu(x), gpu(w), eps=1e-6, out_dtype="f8e4m3")
    ref.check_f8(q[[0, 1, 4, 5]], s[[0, 1, 4, 5]], want[[0, 1, 4, 5]], err[[0, 1, 4, 5]], "f8")
    assert torch.all(s[1] == 1) and torch.isnan(q[2].float()).all()
    # an all-zero row with eps 0 is 0 / 0, as in the formula
    assert torch.isnan(wb.add_rms_norm(gpu(x[1:2]), gpu(w), eps=0.0)[0]).all()


def test_norm_of_tiny_and_huge_values():
    for scale in (1e-30, 1e-18, 1e15):
        x = ref.randn(3, 384, seed=4, dtype="f32", scale=scale)
        w = torch.full((384,), scale)
        q, s, _ = wb.add_rms_norm(gpu(x), gpu(w), eps=0.0 if scale > 1e-20 else 1e-6, out_dtype="f8e4m3")
        want, err, _, _ = ref.norm(x, w, None, 0.0 if scale > 1e-20 else 1e-6)
        if scale == 1e-30:  # everything underflows in fp32: codes of zero
            assert torch.all(q.float() == 0) and torch.all(s == 1)
        else:
            ref.check_f8(q, s, want, err, f"scale {scale}")


# ---- routing -----------------------------------------------------------------------------------

ROUTE_SHAPES = [(1, 1, 1), (1, 8, 2), (3, 2, 2), (17, 8, 2), (64, 60, 4), (65, 16, 3), (130, 17, 17), (200, 64, 6),
                (257, 256, 8), (300, 65, 1), (1000, 8, 2), (70, 513, 20), (33, 1024, 64), (5, 129, 8), (0, 8, 2)]


def routing_inputs(shape, dtype, kind):
    rows, e, k = shape
    z = ref.randn(rows, e, seed=rows + e, dtype="f32", scale=2.0)
    if kind == "ties":
        z = (z * 2).round() / 2
    if kind == "holes":  # experts that are off, and rows of nothing else
        g = torch.Generator().manual_seed(5)
        z[torch.rand(rows, e, generator=g) < 0.5] = -math.inf
        z[::7] = -math.inf
        z[1::7] = torch.finfo(torch.bfloat16).min
    z = z.to(ref.TORCH[dtype])
    mask = None
    if kind in ("masked", "holes"):
        mask = torch.rand(rows, generator=torch.Generator().manual_seed(7)) < 0.7
    if kind == "empty":
        mask = torch.zeros(rows, dtype=torch.bool)
    return z, mask


def check_routing(r, want, shape, what):
    rows, e, k = shape
    for f in ("experts", "positions", "tokens", "counts", "offsets"):
        got = getattr(r, f).cpu().long()
        assert torch.equal(got, want[f]), f"{what}: {f}"
    assert int(r.routed) == want["routed"], what
    # a softmax: exponentials within a few roundings, a sum of e terms
    ref.check(r.gates, want["gates"], want["gates"] * U(e), f"{what}: gates")
    ref.check(r.loss, want["loss"], want["loss"] * (U(e) + U(rows)), f"{what}: loss")


def U(n):
    # exp of an argument up to 2^4 rounded to fp32 is off by up to 2^4 roundings
    return (n + 48) * ref.U32


@pytest.mark.parametrize("kind", ["plain", "ties", "masked", "holes", "empty"])
@pytest.mark.parametrize("shape", ROUTE_SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_route(shape, kind):
    say("route", shape, kind)
    for dtype in ("f32", "bf16"):
        for renormalize in (True, False):
            z, mask = routing_inputs(shape, dtype, kind)
            r = wb.route(gpu(z), shape[2], mask=gpu(mask), renormalize=renormalize)
            check_routing(r, ref.route(z, shape[2], mask, renormalize), shape, f"{dtype} {renormalize}")


def test_route_many_rows():
    """More blocks of rows than one, and more rows than sixty-four in each."""
    z = ref.randn(20011, 12, seed=3, dtype="f32")
    mask = torch.rand(20011, generator=torch.Generator().manual_seed(1)) < 0.9
    shape = (20011, 12, 3)
    want = ref.route(z, 3, mask, True)
    for _ in range(2):
        check_routing(wb.route(gpu(z), 3, mask=gpu(mask)), want, shape, "many")


@pytest.mark.parametrize("kind", ["plain", "ties", "masked", "holes", "empty"])
@pytest.mark.parametrize("shape", ROUTE_SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_route_gradient(shape, kind):
    say("route gradient", shape, kind)
    rows, e, k = shape
    d_gates, d_loss = ref.randn(rows, k, seed=9), 1.7
    for dtype in ("f32", "bf16"):
        for renormalize in (True, False):
            z, mask = routing_inputs(shape, dtype, kind)
            want = ref.route(z, k, mask, renormalize)
            zd = z.double().clone()
            on = (want["experts"] >= 0).any(1)
            zd[~on] = 0
            zd.requires_grad_()
            ref.route_objective(zd, want, k, renormalize, d_gates, d_loss).backward()
            grad = torch.where(on[:, None], zd.grad, torch.zeros_like(zd.grad))
            r = wb.route(gpu(z), k, mask=gpu(mask), renormalize=renormalize)
            got = wb.route_backward(gpu(z), r, gpu(d_gates), torch.tensor([d_loss], device="cuda"))
            assert got.dtype == z.dtype
            # p (dp - sum p dp): within roundings of the magnitudes that meet there
            most = d_gates.abs().sum(1, keepdim=True).double() if rows else torch.zeros(0, 1)
            n = max(1, want["routed"])
            share = d_loss * e * want["counts"].max().double() / (k * n * n)
            p = want["p"] + (want["gates"].amax(1, keepdim=True) if renormalize and k else 0)
            ref.check(got, grad, p * (most + share) * 4 * U(e), f"{dtype} {renormalize}")
            # either part alone
            half = wb.route_backward(gpu(z), r, gpu(d_gates), None).double() + wb.route_backward(
                gpu(z), r, None, torch.tensor([d_loss], device="cuda")).double()
            ref.check(half.float(), grad, (p * (most + share) * 4 * U(e)) + (grad.abs() + p * (most + share)) * 2 * (
                ref.U16 if dtype == "bf16" else ref.U32), "sum of parts")


def test_route_gradient_against_differences():
    rows, e, k = 6, 9, 3
    z = ref.randn(rows, e, seed=2, dtype="f32")
    d_gates = ref.randn(rows, k, seed=3)
    for renormalize in (True, False):
        want = ref.route(z, k, None, renormalize)
        r = wb.route(gpu(z), k, renormalize=renormalize)
        got = wb.route_backward(gpu(z), r, gpu(d_gates), torch.tensor(0.8, device="cuda")).double().cpu()
        h = 1e-5
        for t in range(rows):
            for j in range(e):
                up, down = z.double().clone(), z.double().clone()
                up[t, j] += h
                down[t, j] -= h
                diff = (ref.route_objective(up, want, k, renormalize, d_gates, 0.8)
                        - ref.route_objective(down, want, k, renormalize, d_gates, 0.8)) / (2 * h)
                # the difference itself: h^2 of a third derivative of order one, and 64-bit cancellation
                assert abs(float(got[t, j] - diff)) < 1e-5


def test_route_is_differentiable():
    z = ref.randn(40, 16, seed=2, dtype="bf16").cuda().requires_grad_()
    r = wb.route(z, 4)
    (r.gates.square().sum() + 0.3 * r.loss).backward()
    by_hand = wb.route_backward(z.detach(), r, (2 * r.gates).detach(), torch.tensor([0.3], device="cuda"))
    assert torch.equal(z.grad, by_hand)
    assert not r.experts.requires_grad and not r.counts.requires_grad


def test_route_nan_and_infinity_stay_visible():
    z = ref.randn(80, 8, seed=1, dtype="f32")
    z[3, 2] = math.nan
    z[70, 1] = math.inf
    r = wb.route(gpu(z), 2)
    assert torch.isnan(r.gates[3]).all() and torch.isnan(r.gates[70]).any() and torch.isnan(r.loss)
    assert int(r.experts[70, 0]) == 1 and 2 not in r.experts[3].tolist()
    fine = [t for t in range(80) if t not in (3, 70)]
    want = ref.route(z[fine], 2, None, True)
    assert torch.equal(r.experts[fine].cpu().long(), want["experts"])
    ref.check(r.gates[fine], want["gates"], want["gates"] * U(8), "gates")
    assert int(r.offsets[-1]) == 160 and sorted(r.positions.flatten().tolist()) == list(range(160))


def test_route_strided_logits():
    z = ref.randn(100, 37, seed=1, dtype="bf16")
    a, b = wb.route(gpu(z), 5), wb.route(ref.strided(z, 3, 1), 5)
    for x, y in zip(a[:8], b[:8]):
        assert torch.equal(x, y)


# ---- products ----------------------------------------------------------------------------------

SIZES = [(1, 1, 1), (1, 16, 16), (1, 256, 128), (2, 130, 129), (5, 64, 300), (16, 272, 1000), (17, 96, 64), (33, 640, 384),
         (64, 256, 256), (65, 258, 136), (100, 344, 192), (129, 512, 520), (300, 400, 1504), (1, 1024, 4096)]
FORMS = [dict(), dict(gated=True, activation="silu"), dict(bias=True, activation="gelu", residual=True),
         dict(gated=True, activation="gelu", bias=True, residual=True)]


def product_inputs(rows, n, k, f8, form, seed=0, e=0):
    """Operands on the CPU: x, weight (stacked if e), scales, bias, residual."""
    n = n + n % 2 if form.get("gated") else n
    cols = n // 2 if form.get("gated") else n
    x = ref.randn(rows, k, seed=seed, dtype="bf16")
    w = [ref.randn(n, k, seed=seed + 1 + i, dtype="bf16", scale=k ** -0.5) for i in range(max(1, e))]
    xs = ws = None
    if f8:
        x, xs = ref.quant_rows(x)
        w, ws = zip(*(ref.quant_blocks(m) for m in w))
    b = [ref.randn(n, seed=seed + 70 + i) for i in range(max(1, e))] if form.get("bias") else None
    r = ref.randn(rows, cols, seed=seed + 90, dtype="bf16") if form.get("residual") else None
    return x, w, xs, ws, b, r, cols


def run_linear(x, w, xs, ws, b, r, form, out):
    return wb.linear(x, w, b, x_scales=xs, weight_scales=ws, activation=form.get("activation", "none"),
                     gated=form.get("gated", False), residual=r, out_dtype=out)


def check_product(got, want, err, out, what):
    if out == "f8e4m3":
        if want.shape[0]:
            ref.check_f8(got[0], got[1], want, err, what)
    else:
        assert got.dtype == ref.TORCH[out] and got.shape == want.shape
        ref.check(got, want, err, what)


@pytest.mark.parametrize("f8", [False, True], ids=["bf16", "f8"])
@pytest.mark.parametrize("form", range(len(FORMS)))
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_linear(size, form, f8):
    say("linear", size, FORMS[form], f8)
    form = FORMS[form]
    x, w, xs, ws, b, r, cols = product_inputs(*size, f8, form)
    want, err = ref.product(x, w[0], b and b[0], form.get("activation", "none"), form.get("gated", False), r, xs, ws and ws[0])
    for out in ("bf16", "f32", "f8e4m3"):
        got = run_linear(gpu(x), gpu(w[0]), gpu(xs), gpu(ws and ws[0]), gpu(b and b[0]), gpu(r), form, out)
        torch.cuda.synchronize()
        check_product(got, want, err, out, f"{size} {out}")


@pytest.mark.parametrize("f8", [False, True], ids=["bf16", "f8"])
@pytest.mark.parametrize("size", [(1000, 600, 384), (513, 1024, 1000), (260, 2304, 264), (2100, 520, 512)],
                         ids=lambda s: "x".join(map(str, s)))
def test_linear_of_many_rows(size, f8):
    """Sizes that take the larger tiles."""
    say("linear", size, f8)
    for form in (FORMS[0], FORMS[3]):
        x, w, xs, ws, b, r, cols = product_inputs(*size, f8, form)
        want, err = ref.product(x, w[0], b and b[0], form.get("activation", "none"), form.get("gated", False), r, xs, ws and ws[0])
        for out in ("bf16", "f8e4m3"):
            got = run_linear(gpu(x), gpu(w[0]), gpu(xs), gpu(ws and ws[0]), gpu(b and b[0]), gpu(r), form, out)
            torch.cuda.synchronize()
            check_product(got, want, err, out, f"{size} {out}")


@pytest.mark.parametrize("f8", [False, True], ids=["bf16", "f8"])
@pytest.mark.parametrize("pad,skip", [(0, 1), (3, 0), (16, 16), (5, 7)])
@pytest.mark.parametrize("rows", [1, 20, 200])
def test_linear_of_rows_that_start_anywhere(rows, pad, skip, f8):
    say("linear strided", rows, pad, skip, f8)
    form = FORMS[2]
    x, w, xs, ws, b, r, cols = product_inputs(rows, 144, 272, f8, form)
    want, err = ref.product(x, w[0], b[0], "gelu", False, r, xs, ws and ws[0])
    got = wb.linear(ref.strided(x, pad, skip), ref.strided(w[0], pad, skip), gpu(b[0]),
                    x_scales=ref.strided(xs, 1, 1) if f8 else None, weight_scales=ref.strided(ws[0], 2, 1) if f8 else None,
                    activation="gelu", residual=ref.strided(r, pad, skip), out_dtype="bf16")
    check_product(got, want, err, "bf16", "strided")


def test_linear_reads_scales_of_every_block():
    """Blocks of very different scales: a wrong index would be far off."""
    x, w = ref.randn(40, 700, seed=1), ref.randn(500, 700, seed=2)
    x *= torch.logspace(-3, 3, 6).repeat_interleave(128)[:700]
    w *= torch.logspace(3, -3, 6).repeat_interleave(128)[:700]
    w *= torch.logspace(-2, 2, 4).repeat_interleave(128)[:500, None]
    (x, xs), (w, ws) = ref.quant_rows(x), ref.quant_blocks(w)
    for gated in (False, True):
        want, err = ref.product(x, w, None, "silu", gated, None, xs, ws)
        check_product(wb.linear(gpu(x), gpu(w), x_scales=gpu(xs), weight_scales=gpu(ws), activation="silu", gated=gated,
                                out_dtype="f32"), want, err, "f32", f"gated {gated}")


def test_linear_keeps_nan_to_its_row_and_column():
    x, w = ref.randn(70, 200, seed=1, dtype="bf16"), ref.randn(300, 200, seed=2, dtype="bf16")
    x[69, 3] = math.nan
    w[299, 7] = math.inf
    got = wb.linear(gpu(x), gpu(w), out_dtype="f32")
    assert torch.isnan(got[69]).all() and not torch.isfinite(got[:, 299]).any()
    want, err = ref.product(x[:69], w[:299], None, "none", False, None)
    ref.check(got[:69, :299], want, err, "the others")


# ---- products with stacked weights -------------------------------------------------------------

COUNTS = [[3], [0, 5, 0], [1, 1, 1, 1], [70, 0, 3, 129, 1], [0, 0, 0], [2] * 70, [300, 20]]


@pytest.mark.parametrize("f8", [False, True], ids=["bf16", "f8"])
@pytest.mark.parametrize("gather", [False, True], ids=["rows", "tokens"])
@pytest.mark.parametrize("counts", range(len(COUNTS)))
def test_expert_linear(counts, gather, f8):
    counts = COUNTS[counts]
    say("experts", counts, gather, f8)
    e, rows = len(counts), sum(counts)
    for (n, k), form in zip([(256, 128), (130, 200), (96, 272)], [FORMS[1], FORMS[2], FORMS[3]]):
        x, w, xs, ws, b, r, cols = product_inputs(rows, n, k, f8, form, e=e)
        tokens = None
        if gather:
            tokens = torch.randint(0, max(1, rows), (rows,), generator=torch.Generator().manual_seed(3), dtype=torch.int32)
        at = [0]
        for c in counts:
            at.append(at[-1] + c)
        wants, errs = [], []
        for i in range(e):
            mine = slice(at[i], at[i + 1])
            from_ = tokens[mine].long() if gather else mine
            want, err = ref.product(x[from_], w[i], b and b[i], form["activation"], form.get("gated", False),
                                    None if r is None else r[mine], None if xs is None else xs[from_], ws and ws[i])
            wants.append(want)
            errs.append(err)
        for out in ("bf16", "f8e4m3"):
            got = wb.expert_linear(gpu(x), torch.stack(w).cuda(), torch.tensor(at, dtype=torch.int32, device="cuda"),
                                   gpu(tokens), torch.stack(b).cuda() if b else None, x_scales=gpu(xs),
                                   weight_scales=torch.stack(ws).cuda() if f8 else None, activation=form["activation"],
                                   gated=form.get("gated", False), residual=gpu(r), out_dtype=out)
            torch.cuda.synchronize()
            check_product(got, torch.cat(wants), torch.cat(errs), out, f"{counts} {n} {k} {out}")


def test_expert_linear_leaves_other_ranks_rows():
    """A rank's slice of the offsets: rows before and behind it stay as they
    were, and offsets past the rows are cut off."""
    lib, n, k = wb.lib, 64, 64
    x, w = ref.randn(50, k, seed=1, dtype="bf16").cuda(), ref.randn(3, n, k, seed=2, dtype="bf16").cuda()
    full = wb.expert_linear(x, w, torch.tensor([0, 20, 30, 50], dtype=torch.int32, device="cuda"))
    for lo, a, b, hi in ((10, 20, 30, 44), (0, 0, 30, 1000), (-5, 20, 10, 30)):
        out = torch.full((50, n), 7.0, dtype=torch.bfloat16, device="cuda")
        got = out.clone()
        args = ref_args(x, w, got, torch.tensor([lo, a, b, hi], dtype=torch.int32, device="cuda"))
        assert lib.wb_linear(args[0], None, ctypes.c_size_t(0), None) == 0, lib.wb_last_error()
        torch.cuda.synchronize()
        first, last = max(lo, 0), min(hi, 50)
        assert torch.all(got[:first] == 7) and torch.all(got[last:] == 7)
        if (lo, a, b, hi) == (10, 20, 30, 44):
            assert torch.equal(got[20:30], full[20:30]) and torch.equal(got[30:44], full[30:44])
            assert torch.equal(got[10:20], full[10:20])


def ref_args(x, w, out, offsets):
    class Matrix(ctypes.Structure):
        _fields_ = [("data", ctypes.c_void_p), ("dtype", ctypes.c_int32), ("reserved", ctypes.c_int32),
                    ("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("ld", ctypes.c_int64)]

    class Args(ctypes.Structure):
        _fields_ = [(f, Matrix) for f in ("x", "x_scales", "weight", "weight_scales", "bias", "residual", "out", "out_scales")]
        _fields_ += [("offsets", ctypes.c_void_p), ("tokens", ctypes.c_void_p), ("num_experts", ctypes.c_int32),
                     ("activation", ctypes.c_int32), ("gated", ctypes.c_int32), ("reserved", ctypes.c_int32)]

    a = Args()
    a.x = Matrix(x.data_ptr(), 1, 0, *x.shape, x.shape[1])
    a.weight = Matrix(w.data_ptr(), 1, 0, w.shape[0] * w.shape[1], w.shape[2], w.shape[2])
    a.out = Matrix(out.data_ptr(), 1, 0, *out.shape, out.shape[1])
    a.offsets, a.num_experts = offsets.data_ptr(), w.shape[0]
    return ctypes.byref(a), a, offsets


# ---- sums of expert rows -----------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 1, 1), (3, 7, 2), (5, 2048, 8), (20, 2056, 3), (4, 4099, 64), (0, 16, 2)],
                         ids=lambda s: "x".join(map(str, s)))
def test_combine(shape, dtype):
    say("combine", shape, dtype)
    rows, cols, k = shape
    n = max(1, rows * k)
    y = ref.randn(n, cols, seed=1, dtype=dtype)
    g = torch.Generator().manual_seed(2)
    pos = torch.randint(-2, n + 2, (rows, k), generator=g, dtype=torch.int32)
    gates = ref.randn(rows, k, seed=3)
    for residual in (None, ref.randn(rows, cols, seed=4, dtype="bf16")):
        for span in (None, (0, n), (n // 3, n // 2), (5, 5)):
            lo, hi = span or (0, n)
            there = ((pos >= max(0, lo)) & (pos < min(hi, n))).double()
            rows_of = y.double()[pos.long().clamp(0, n - 1)]
            want = (rows_of * (gates.double() * there)[..., None]).sum(1)
            err = (rows_of.abs() * (gates.double() * there).abs()[..., None]).sum(1) * ref.U32 * (k + 2)
            if residual is not None:
                want = want + residual.double()
                err = err + want.abs() * ref.U32
            offs = torch.tensor([span[0], 1, 2, span[1]], dtype=torch.int32, device="cuda") if span else None
            for out in ("f32", "bf16"):
                got = wb.combine(gpu(y), gpu(pos), gpu(gates), residual=gpu(residual), span=offs, out_dtype=out)
                assert got.dtype == ref.TORCH[out]
                ref.check(got, want, err, f"{shape} {span} {out}")


def test_combine_skips_what_unused_places_hold():
    y = torch.full((8, 64), math.nan, device="cuda")
    y[2] = 1.0
    pos = torch.tensor([[2, -1], [-1, -1], [2, 9]], dtype=torch.int32, device="cuda")
    gates = torch.tensor([[0.5, math.inf], [math.nan, 1.0], [0.25, 1.0]], device="cuda")
    got = wb.combine(y, pos, gates)
    assert torch.all(got[0] == 0.5) and torch.all(got[1] == 0) and torch.all(got[2] == 0.25)


# ---- together, and around ----------------------------------------------------------------------

def test_operators_on_a_stream_of_their_own():
    x, w = ref.randn(300, 512, seed=1, dtype="bf16").cuda(), ref.randn(256, 512, seed=2, dtype="bf16").cuda()
    g = torch.ones(512, dtype=torch.bfloat16, device="cuda")
    z = ref.randn(300, 16, seed=3).cuda()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    q, sc, _ = wb.add_rms_norm(x, g, out_dtype="f8e4m3", stream=s)
    y = wb.linear(x, w, stream=s)
    r = wb.route(z, 4, stream=s)
    d = wb.route_backward(z, r, torch.ones_like(r.gates), stream=s)
    c = wb.combine(y, r.positions % 300, r.gates, stream=s.cuda_stream)
    s.synchronize()
    q0, sc0, _ = wb.add_rms_norm(x, g, out_dtype="f8e4m3")
    r0 = wb.route(z, 4)
    assert torch.equal(q.view(torch.uint8), q0.view(torch.uint8)) and torch.equal(sc, sc0)
    assert torch.equal(y, wb.linear(x, w))
    assert all(torch.equal(a, b) for a, b in zip(r[:8], r0[:8]))
    assert torch.equal(d, wb.route_backward(z, r0, torch.ones_like(r0.gates)))
    assert torch.equal(c, wb.combine(wb.linear(x, w), r0.positions % 300, r0.gates))


def test_operators_in_a_graph():
    """Captured once, replayed on new inputs with eager work in between."""
    x, z = ref.randn(40, 256, seed=1, dtype="bf16").cuda(), ref.randn(40, 8, seed=2).cuda()
    w = ref.randn(8, 128, 256, seed=3, dtype="bf16").cuda()
    g = torch.ones(256, dtype=torch.bfloat16, device="cuda")

    def layer():
        h, _, _ = wb.add_rms_norm(x, g)
        r = wb.route(z, 2)
        y = wb.expert_linear(h, w, r.offsets, tokens=r.tokens, activation="silu", gated=True)
        return wb.combine(y, r.positions, r.gates), r.loss

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, loss = layer()
    for i in range(4):
        x.copy_(ref.randn(40, 256, seed=10 + i, dtype="bf16"))
        z.copy_(ref.randn(40, 8, seed=20 + i))
        graph.replay()
        torch.cuda.synchronize()
        want, want_loss = layer()
        assert torch.equal(out, want) and torch.equal(loss, want_loss), i


def test_results_do_not_change_from_call_to_call():
    z = ref.randn(5000, 64, seed=1).cuda()
    x, w = ref.randn(700, 640, seed=2, dtype="bf16").cuda(), ref.randn(512, 640, seed=3, dtype="bf16").cuda()
    first = wb.route(z, 6), wb.linear(x, w, out_dtype="f32")
    for _ in range(5):
        again = wb.route(z, 6), wb.linear(x, w, out_dtype="f32")
        assert all(torch.equal(a, b) for a, b in zip(first[0][:8], again[0][:8])) and torch.equal(first[1], again[1])


def test_refusals():
    f = lambda *s, dt=torch.bfloat16: torch.zeros(*s, dtype=dt, device="cuda")  # noqa: E731
    i = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    x, w, v = f(4, 64), f(32, 64), f(64)
    f8 = torch.float8_e4m3fn
    bad = [
        lambda: wb.add_rms_norm(x.cpu(), v), lambda: wb.add_rms_norm(x, v[:63]), lambda: wb.add_rms_norm(x, v, f(4, 63)),
        lambda: wb.add_rms_norm(x, v, eps=-1.0), lambda: wb.add_rms_norm(x, v, out_dtype="f16"),
        lambda: wb.add_rms_norm(x.half(), v), lambda: wb.add_rms_norm(x[0], v), lambda: wb.add_rms_norm(x.t(), f(4)),
        lambda: wb.add_rms_norm(f(4, 64, dt=f8), v), lambda: wb.add_rms_norm(x, v, eps=math.nan),
        lambda: wb.route(x, 0), lambda: wb.route(x, 65), lambda: wb.route(f(4, 1025), 2), lambda: wb.route(f(4, 100), 65),
        lambda: wb.route(x, 2, mask=f(4)), lambda: wb.route(x, 2, mask=f(3, dt=torch.bool)), lambda: wb.route(v, 2),
        lambda: wb.route_backward(x, wb.route(x, 2), f(4, 2)), lambda: wb.route_backward(f(5, 64), wb.route(x, 2)),
        lambda: wb.linear(x, f(32, 63)), lambda: wb.linear(x, w.float()), lambda: wb.linear(x.float(), w.float()),
        lambda: wb.linear(x, w, activation="tanh"), lambda: wb.linear(x, f(31, 64), gated=True),
        lambda: wb.linear(x, w, residual=f(4, 31)), lambda: wb.linear(x, w, f(31)), lambda: wb.linear(x, w, out_dtype=None),
        lambda: wb.linear(x, w, x_scales=f(4, 1, dt=torch.float32)), lambda: wb.linear(x.to(f8), w.to(f8)),
        lambda: wb.linear(x.to(f8), w.to(f8), x_scales=f(4, 1, dt=torch.float32), weight_scales=f(2, 1, dt=torch.float32)),
        lambda: wb.linear(x, w.t().contiguous().t()), lambda: wb.linear(x, f(2, 16, 64)),
        lambda: wb.expert_linear(x, f(2, 16, 64), None), lambda: wb.expert_linear(x, f(2, 16, 64), i(0, 4)),
        lambda: wb.expert_linear(x, f(2, 16, 64), i(0, 2, 4).long()),
        lambda: wb.expert_linear(x, f(2, 16, 64), i(0, 2, 4), tokens=i(0, 1).long()),
        lambda: wb.expert_linear(x, f(2, 16, 64), i(0, 2, 4), bias=f(16)),
        lambda: wb.expert_linear(x, f(2, 32, 64)[:, :16], i(0, 2, 4)),
        lambda: wb.combine(x, i(0, 1), f(2, dt=torch.float32)), lambda: wb.combine(x, f(2, 2), f(2, 2, dt=torch.float32)),
        lambda: wb.combine(x, i(0, 1).view(2, 1), f(2, 2, dt=torch.float32)),
        lambda: wb.combine(x, i(0, 1).view(2, 1), f(2, 1, dt=torch.float32), residual=f(3, 64)),
        lambda: wb.combine(x, f(2, 65, dt=torch.int32), f(2, 65, dt=torch.float32)),
        lambda: wb.combine(x, i(0, 1).view(2, 1), f(2, 1, dt=torch.float32), out_dtype="f8e4m3"),
    ]
    for n, call in enumerate(bad):
        with pytest.raises(wb.WbError) as e:
            call()
        assert str(e.value), n
    torch.cuda.synchronize()


# ---- rows off the 16-byte grid that are copied onto it first ------------------------------------

@pytest.mark.parametrize("f8", [False, True], ids=["bf16", "f8"])
@pytest.mark.parametrize("size", [(2, 1337, 7543), (8, 96, 6001), (300, 1000, 1501), (1000, 1056, 1001), (1030, 2304, 250)],
                         ids=lambda s: "x".join(map(str, s)))
def test_linear_of_long_or_many_odd_rows(size, f8):
    say("linear copied", size, f8)
    for form in (FORMS[0], FORMS[3]) if size[1] % 32 == 0 else (FORMS[0],):
        x, w, xs, ws, b, r, cols = product_inputs(*size, f8, form)
        want, err = ref.product(x, w[0], b and b[0], form.get("activation", "none"), form.get("gated", False), r, xs, ws and ws[0])
        for out in ("f32", "f8e4m3"):
            got = run_linear(gpu(x), gpu(w[0]), gpu(xs), gpu(ws and ws[0]), gpu(b and b[0]), gpu(r), form, out)
            torch.cuda.synchronize()
            check_product(got, want, err, out, f"{size} {out}")


@pytest.mark.parametrize("f8", [False, True], ids=["bf16", "f8"])
@pytest.mark.parametrize("which", ["x", "weight", "both"])
def test_linear_copies_only_what_is_off_the_grid(which, f8):
    """Values beyond the rows' ends are NaN: a copy must not take them along."""
    say("linear copied", which, f8)
    x, w, xs, ws, _, _, _ = product_inputs(24, 96, 6016, f8, {})
    want, err = ref.product(x, w[0], None, "none", False, None, xs, ws and ws[0])

    def off(t):
        wide = torch.full((t.shape[0], t.shape[1] + 24), math.nan).to(t.dtype).cuda()
        wide[:, 5:5 + t.shape[1]] = gpu(t)
        return wide[:, 5:5 + t.shape[1]]

    gx = gpu(x) if which == "weight" else off(x)
    gw = gpu(w[0]) if which == "x" else off(w[0])
    got = wb.linear(gx, gw, x_scales=gpu(xs), weight_scales=gpu(ws and ws[0]), out_dtype="f32")
    torch.cuda.synchronize()
    ref.check(got, want, err, which)


@pytest.mark.parametrize("f8", [False, True], ids=["bf16", "f8"])
def test_expert_linear_of_long_odd_rows(f8):
    say("experts copied", f8)
    counts, n, k = [1, 0, 40, 23], 64, 4111
    x, w, xs, ws, _, _, _ = product_inputs(30, n, k, f8, {}, e=len(counts))
    tokens = torch.arange(sum(counts), dtype=torch.int32) % 30
    at, wants, errs = [0], [], []
    for i, c in enumerate(counts):
        mine = tokens[at[-1]:at[-1] + c].long()
        at.append(at[-1] + c)
        want, err = ref.product(x[mine], w[i], None, "none", False, None, None if xs is None else xs[mine], ws and ws[i])
        wants.append(want)
        errs.append(err)
    got = wb.expert_linear(gpu(x), torch.stack(w).cuda(), torch.tensor(at, dtype=torch.int32, device="cuda"), gpu(tokens),
                           x_scales=gpu(xs), weight_scales=torch.stack(ws).cuda() if f8 else None, out_dtype="f32")
    torch.cuda.synchronize()
    ref.check(got, torch.cat(wants), torch.cat(errs), "experts")


# ---- integers that are no expert's number --------------------------------------------------------

@pytest.mark.parametrize("shape", [(40, 8, 4), (70, 60, 17), (33, 256, 8), (9, 513, 20)], ids=lambda s: "x".join(map(str, s)))
def test_route_gradient_leaves_out_choices_that_are_no_experts(shape):
    """As if they were -1, bit for bit, in their own row and in its neighbours."""
    say("route gradient, experts out of range", shape)
    rows, e, k = shape
    z = ref.randn(rows, e, seed=4).cuda()
    d_gates, d_loss = ref.randn(rows, k, seed=5).cuda(), torch.tensor(0.5, device="cuda")
    away = torch.rand(rows, k, generator=torch.Generator().manual_seed(6)).cuda() < 0.4
    wrong = torch.tensor([e, e + 1, 2 * e, 1023, 1024, 1 << 20, 2 ** 31 - 1, -2, -2 ** 31], dtype=torch.int32, device="cuda")
    wrong = wrong[(wrong < 0) | (wrong >= e)]
    for renormalize in (True, False):
        r = wb.route(z, k, renormalize=renormalize)
        some = wrong[torch.arange(rows * k, device="cuda") % wrong.numel()].view(rows, k)
        got = wb.route_backward(z, r._replace(experts=torch.where(away, some, r.experts)), d_gates, d_loss)
        want = wb.route_backward(z, r._replace(experts=torch.where(away, torch.full_like(some, -1), r.experts)), d_gates, d_loss)
        assert torch.equal(got, want), renormalize


# ---- operators without a gradient ---------------------------------------------------------------

def test_operators_without_a_gradient_refuse_tensors_that_require_one():
    """A result without a graph would lose the gradient silently."""
    f = lambda *s: torch.ones(*s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    need = lambda t: t.detach().clone().requires_grad_()  # noqa: E731
    x, w, g, r, b = f(4, 64), f(32, 64), f(64), f(4, 64), f(32)
    f8, xs, ws = torch.float8_e4m3fn, torch.ones(4, 1, device="cuda"), torch.ones(1, 1, device="cuda")
    stacked, at = f(2, 32, 64), torch.tensor([0, 2, 4], dtype=torch.int32, device="cuda")
    routing = wb.route(torch.randn(2, 8, device="cuda").requires_grad_(), 2)
    assert routing.gates.requires_grad
    z, plain = torch.randn(2, 8, device="cuda"), routing.gates.detach()
    codes = lambda **k: wb.linear(x.to(f8), w.to(f8), **{"x_scales": xs, "weight_scales": ws, **k})  # noqa: E731
    calls = [
        lambda: wb.add_rms_norm(need(x), g), lambda: wb.add_rms_norm(x, need(g)), lambda: wb.add_rms_norm(x, g, need(r)),
        lambda: wb.linear(need(x), w), lambda: wb.linear(x, need(w)), lambda: wb.linear(x, w, need(b)),
        lambda: wb.linear(x, w, residual=need(f(4, 32))), lambda: codes(x_scales=need(xs)),
        lambda: codes(weight_scales=need(ws)), lambda: wb.expert_linear(x, need(stacked), at),
        lambda: wb.expert_linear(need(x), stacked, at), lambda: wb.combine(x, routing.positions, routing.gates),
        lambda: wb.combine(need(x), routing.positions, plain),
        lambda: wb.combine(x, routing.positions, plain, residual=need(f(2, 64))),
        lambda: wb.route_backward(z, routing, need(plain)),
        lambda: wb.route_backward(z, routing, plain, need(torch.ones((), device="cuda"))),
    ]
    for n, call in enumerate(calls):
        with pytest.raises(wb.WbError, match="requires a gradient"):
            call()
        with torch.no_grad():
            call()
    # tensors that are part of no graph, and the router's own way back
    wb.combine(x, routing.positions, routing.gates.detach())
    wb.route_backward(need(z), routing, plain)
    torch.cuda.synchronize()


def test_operators_refuse_forward_mode_tangents():
    import torch.autograd.forward_ad as fw

    z, x, w, g = torch.randn(2, 8, device="cuda"), *(torch.ones(*s, dtype=torch.bfloat16, device="cuda") for s in ((2, 64), (32, 64), (64,)))
    r = wb.route(z, 2)
    with fw.dual_level():
        dual = lambda t: fw.make_dual(t, torch.ones_like(t))  # noqa: E731
        for n, call in enumerate([
                lambda: wb.route(dual(z), 2), lambda: wb.route(dual(z.clone().requires_grad_()), 2),
                lambda: wb.route_backward(dual(z), r, r.gates), lambda: wb.route_backward(z, r, dual(r.gates)),
                lambda: wb.add_rms_norm(dual(x), g), lambda: wb.linear(x, dual(w)),
                lambda: wb.combine(x, r.positions, dual(r.gates))]):
            with pytest.raises(wb.WbError, match="tangent"):
                call()
        assert fw.unpack_dual(wb.route(z, 2).gates).tangent is None
    wb.route(z, 2)
    torch.cuda.synchronize()


# ---- fp8 results among the smallest numbers ------------------------------------------------------

def test_fp8_results_of_subnormal_scales_are_no_nan():
    """608 units of 2^-149 have a scale of 1.36 of them, one when rounded: their quotients are past E4M3's
    largest, and are held to it."""
    unit = 2.0 ** -149
    w = torch.zeros(128, dtype=torch.float64)
    w[:6] = torch.tensor([608.0, -608.0, 288.0, 97.0, -3.0, 1.0])
    want = torch.tensor([448.0, -448.0, 288.0, 96.0, -3.0, 1.0])
    x = torch.ones(3, 128, device="cuda")
    x[1, 7] = math.nan
    q, s, _ = wb.add_rms_norm(x, (w * unit).float().cuda(), eps=0.0, out_dtype="f8e4m3")
    for t in (0, 2):  # y is the weight itself
        assert float(s[t, 0]) == unit and torch.equal(q[t].float().cpu()[:6], want), q[t, :6].float()
        assert torch.all(q[t, 6:].float() == 0)
    assert torch.isnan(q[1].float()).all()
    # the same as sums of two products of codes, few rows and many
    f8 = torch.float8_e4m3fn
    codes = torch.zeros(256, 128)
    codes[:6, :2] = torch.tensor([[448.0, 160.0], [-448.0, -160.0], [288.0, 0.0], [96.0, 1.0], [-3.0, 0.0], [1.0, 0.0]])
    for rows in (1, 700, 9000):
        a = torch.zeros(rows, 128)
        a[:, :2] = 1.0
        got, gs = wb.linear(a.to(f8).cuda(), codes.to(f8).cuda(), x_scales=torch.full((rows, 1), 2.0 ** -75, device="cuda"),
                            weight_scales=torch.full((2, 1), 2.0 ** -74, device="cuda"), out_dtype="f8e4m3")
        assert torch.all(gs[:, 0] == unit) and torch.all(gs[:, 1] == 1.0), rows
        assert torch.equal(got[:, :6].float().cpu(), want.expand(rows, 6)) and torch.all(got[:, 6:].float() == 0), rows


# ---- roundings of the activations and of the router ----------------------------------------------

@pytest.mark.parametrize("k", [1, 16], ids=["registers", "direct"])
def test_silu_is_within_a_few_roundings(k):
    """z itself is exact (one product by one). Roundings of half a unit: e^-|z| three (the instruction's unit and a
    sum), 1 + t one and at most half of the three, its reciprocal one, z t one more, their product one: nine."""
    z = torch.cat([torch.linspace(-85, 88, 4001), torch.logspace(-30, 1.9, 2001), -torch.logspace(-30, 1.9, 2001)]).bfloat16()
    w, x = torch.zeros(z.numel(), k, dtype=torch.bfloat16), torch.zeros(2, k, dtype=torch.bfloat16)
    w[:, 0], x[:, 0] = z, 1.0
    got = wb.linear(gpu(x), gpu(w), activation="silu", out_dtype="f32").double().cpu()
    want = z.double() * torch.sigmoid(z.double())
    off = ((got - want).abs() - 9 * ref.U32 * want.abs()).amax(0)
    assert float(off.max()) <= 0, (float(z[off.argmax()]), float((got - want).abs().amax(0)[off.argmax()] / want.abs()[off.argmax()] / ref.U32))
    # gated, by an up of one
    both = torch.cat([w, w])
    both[z.numel():, 0] = 1.0
    assert torch.equal(wb.linear(gpu(x), gpu(both), activation="silu", gated=True, out_dtype="f32").double().cpu(), got)


def test_silu_of_the_ends():
    z = torch.tensor([0.0, -0.0, 100.0, 3e38, math.inf, -100.0, -200.0, -3e38, math.nan]).bfloat16()
    w = torch.zeros(z.numel(), 16, dtype=torch.bfloat16)
    w[:, 0] = z
    x = torch.zeros(1, 16, dtype=torch.bfloat16)
    x[0, 0] = 1.0
    w[4, 1:], w[8, 1:] = 0.0, 0.0
    got = wb.linear(gpu(x), gpu(w), activation="silu", out_dtype="f32")[0].cpu()
    assert torch.equal(got[:2], torch.zeros(2)) and torch.equal(got[2:5], z[2:5].float())
    assert torch.all(got[5:8].abs() <= 1e-38) and torch.isnan(got[8])


@pytest.mark.parametrize("experts,k", [(8, 2), (8, 8), (64, 6), (256, 8), (1024, 8)])
@pytest.mark.parametrize("renormalize", [True, False])
def test_gates_and_gradient_are_off_by_no_more_than_the_formula_in_fp32(experts, k, renormalize):
    """A gate takes the roundings of an exponential, of a sum and of a quotient, as elementary operations in fp32 do:
    their root mean squares over 20000 rows are the same but for 0.5 % of spread in each, 3 % being four of both."""
    say("roundings", experts, k, renormalize)
    g = torch.Generator(device="cuda").manual_seed(experts + k)
    rows = 20000
    z = torch.randn(rows, experts, generator=g, device="cuda") * 1.5
    d_gates, d_loss = torch.randn(rows, k, generator=g, device="cuda"), torch.tensor(0.7 * rows, device="cuda")
    r = wb.route(z, k, renormalize=renormalize)
    at = r.experts.long()

    def formula(z, type):
        top = z.amax(1, keepdim=True)
        e = torch.exp(z - top)
        p = e / e.sum(1, keepdim=True)
        gates = e.gather(1, at)
        gates = gates / (gates if renormalize else e).sum(1, keepdim=True)
        dg = d_gates.to(type)
        dp = (r.counts.to(type) * (experts / (k * rows * rows)) * d_loss.to(type)).expand(rows, experts)
        if not renormalize:
            dp = dp.scatter_add(1, at, dg)
        d = p * (dp - (p * dp).sum(1, keepdim=True))
        if renormalize:
            d = d.scatter_add(1, at, gates * (dg - (dg * gates).sum(1, keepdim=True)))
        return gates, d

    want, plain = formula(z.double(), torch.float64), formula(z, torch.float32)
    got = r.gates, wb.route_backward(z, r, d_gates, d_loss)
    rms = lambda a, w: float(((a.double() - w) / w).square().mean().sqrt())  # noqa: E731
    assert rms(got[0], want[0]) <= 1.03 * rms(plain[0], want[0]), "gates"
    off = lambda a: float((a.double() - want[1]).norm())  # noqa: E731
    assert off(got[1]) <= 1.03 * off(plain[1]), "gradient"


# ---- rows that 32-bit offsets do not reach --------------------------------------------------------

def far(t, apart):
    """The same values with rows ``apart`` elements from each other, in memory that is otherwise left as it is."""
    rows, cols = t.shape
    view = torch.empty((rows - 1) * apart + cols, dtype=t.dtype, device="cuda").as_strided((rows, cols), (apart, 1))
    view.copy_(gpu(t))
    return view


@pytest.mark.parametrize("f8", [False, True], ids=["bf16", "f8"])
@pytest.mark.parametrize("which", ["x", "weight", "gathered x"])
def test_products_of_rows_far_apart(which, f8):
    """Past 2^32 bytes from the first row to the last: the offsets in registers are 32 bits wide."""
    say("linear far", which, f8)
    apart = (1 << 24) // (1 if f8 else 2)  # 16 MiB
    x, w, xs, ws, b, r, cols = product_inputs(300, 288, 208, f8, FORMS[2])
    gx, gw = (gpu(x), far(w[0], apart)) if which == "weight" else (far(x, apart), gpu(w[0]))
    more = dict(x_scales=gpu(xs), weight_scales=gpu(ws and ws[0]), activation="gelu", residual=gpu(r), out_dtype="f32")
    if which == "gathered x":
        tokens = (torch.arange(300, dtype=torch.int32) * 7 + 290) % 300
        at = torch.tensor([0, 300], dtype=torch.int32, device="cuda")
        got = wb.expert_linear(gx, gw[None], at, gpu(tokens), gpu(b[0])[None], **{**more, "weight_scales": ws and gpu(ws[0])[None]})
        x, xs = x[tokens.long()], None if xs is None else xs[tokens.long()]
    else:
        got = wb.linear(gx, gw, gpu(b[0]), **more)
    want, err = ref.product(x, w[0], b[0], "gelu", False, r, xs, ws and ws[0])
    ref.check(got, want, err, which)


def test_stacked_weights_past_four_gigabytes():
    """Each expert's rows start past 32 bits from the first expert's; within an expert they are near."""
    say("experts far")
    apart, n, k, e = 1 << 21, 96, 128, 25  # 4 MiB a row, 9.4 GiB in all
    w = ref.randn(n * e, k, seed=3, dtype="bf16", scale=k ** -0.5)
    x = ref.randn(2 * e, k, seed=4, dtype="bf16")
    stacked = far(w, apart).unflatten(0, (e, n))
    at = torch.arange(0, 2 * e + 1, 2, dtype=torch.int32)
    got = wb.expert_linear(gpu(x), stacked, gpu(at), out_dtype="f32")
    parts = [ref.product(x[2 * i:2 * i + 2], w[n * i:n * i + n], None, "none", False, None) for i in range(e)]
    ref.check(got, torch.cat([p[0] for p in parts]), torch.cat([p[1] for p in parts]), "experts")


def test_norm_sum_and_routing_of_rows_far_apart():
    say("rows far")
    apart = 1 << 22
    x, r, w = ref.randn(600, 300, seed=1, dtype="f32"), ref.randn(600, 300, seed=2, dtype="bf16"), ref.randn(300, seed=3)
    for out in ("bf16", "f8e4m3"):
        got = wb.add_rms_norm(far(x, apart), gpu(w), far(r, apart), out_dtype=out)
        want = wb.add_rms_norm(gpu(x), gpu(w), gpu(r), out_dtype=out)
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(got, want) if a is not None)
    pos = torch.randperm(1200, generator=torch.Generator().manual_seed(1)).view(600, 2).int() % 600
    gates = ref.randn(600, 2, seed=5)
    assert torch.equal(wb.combine(far(x, apart), gpu(pos), gpu(gates), residual=far(r, apart)),
                       wb.combine(gpu(x), gpu(pos), gpu(gates), residual=gpu(r)))
    a, b = wb.route(far(x, apart), 6), wb.route(gpu(x), 6)
    assert all(torch.equal(u, v) for u, v in zip(a[:8], b[:8]))
    assert torch.equal(wb.route_backward(far(x, apart), a, torch.ones_like(a.gates)), wb.route_backward(gpu(x), b, torch.ones_like(b.gates)))


def test_route_has_no_second_derivative_and_says_so():
    z = torch.randn(6, 8, generator=torch.Generator().manual_seed(1)).cuda().requires_grad_()
    first, = torch.autograd.grad(wb.route(z, 2).loss, z)
    r = wb.route(z, 2)
    d, = torch.autograd.grad(r.loss, z, create_graph=True)
    assert torch.equal(d, first) and d.requires_grad
    with pytest.raises(wb.WbError, match="no gradient of its own"):
        (z.sum() + d.square().sum()).backward()
    r = wb.route(z, 2)
    weight = torch.ones(6, 2, device="cuda", requires_grad=True)
    d, = torch.autograd.grad((r.gates * weight).sum(), z, create_graph=True)
    with pytest.raises(wb.WbError, match="no gradient of its own"):
        d.square().sum().backward()


@pytest.mark.parametrize("rows", [1, 40, 100])
def test_an_infinite_scale_of_the_last_block_gives_infinities(rows):
    """An odd number of blocks of 128, which tiles take two or four at a time: nothing is added for those past the end."""
    f8, inf = torch.float8_e4m3fn, math.inf
    for k in (128, 384, 640, 141, 400):
        nb = ref.blocks(k)
        x, w = torch.ones(rows, k).to(f8).cuda(), torch.ones(64, k).to(f8).cuda()
        xs, ws = torch.ones(rows, nb, device="cuda"), torch.ones(1, nb, device="cuda")
        xs[rows - 1, nb - 1] = inf
        got = wb.linear(x, w, x_scales=xs, weight_scales=ws, out_dtype="f32")
        assert torch.all(got[rows - 1] == inf) and torch.all(got[:rows - 1] == k), k
        ws[0, nb - 1] = 1e30  # 1e30 twice is infinite as well
        xs[rows - 1, nb - 1] = 1e30
        got = wb.linear(x, w, x_scales=xs, weight_scales=ws, out_dtype="f32")
        assert torch.all(got[rows - 1] == inf) and torch.isfinite(got[:rows - 1]).all(), k


def test_a_result_that_memory_does_not_hold_is_torch_s_own_error():
    """70 TB: programs that make room and try again wait for this type."""
    x, w = torch.zeros(1 << 21, 8, dtype=torch.bfloat16, device="cuda"), torch.zeros(1 << 24, 8, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(torch.OutOfMemoryError):
        wb.linear(x, w)
    assert torch.all(wb.linear(x[:16], w[:16]) == 0)
