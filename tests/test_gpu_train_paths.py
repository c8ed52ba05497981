"""The trainer's operators at the sizes that take their kernels' other paths:
gradients of the norm over several turns of every width and in memory that it
replaces, gradients of other types than what they are of, and launches that go
past the caches, with rows off the vectors' grid."""

import ctypes
import math

import pytest
import torch

import ops_ref as ref
import paper_2609_25442_amd as wb
import train_ref as tr
from gpu_util import say

pytestmark = pytest.mark.gpu
T = ref.TORCH


def draw(rows, cols, seed, dtype):
    """Values as ref.randn's, made on the GPU: for large ones."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(rows, cols, generator=g, device="cuda").to(T[dtype])


def against_formula(x, w, b, r, d, more, center, eps=1e-3):
    """A norm and its gradient against the formulas in 64 bits."""
    n = wb.add_layer_norm(x, w, b, r, eps=eps, center=center)
    host = lambda t: None if t is None else t.cpu()  # noqa: E731
    f = tr.layer_norm(host(x), host(w), host(b), host(r), float(torch.tensor(eps)), center)
    assert torch.equal(n.total.cpu(), f["total"])
    ref.check(n.out, f["out"], f["e_out"], "norm")
    got = wb.add_layer_norm_backward(d, n, w, d_total=more)
    of_sum, of_w, of_b = tr.layer_norm_backward(f, host(w), host(d), host(more), center)
    ref.check(got.x, *of_sum, "gradient of x")
    if r is not None:
        ref.check(got.residual, *of_sum, "gradient of the residual")
    ref.check(got.weight, *of_w, "gradient of the weight")
    if b is not None:
        ref.check(got.bias, *of_b, "gradient of the bias")
    return n, got


# a workgroup's rows: eight of one wavefront, four of two, two of four, one of eight; 256 or 512 workgroups
TURNS = [(5000, 136), (2500, 520), (1100, 1000), (1777, 1501), (1300, 2048), (600, 2050), (1200, 3001), (600, 4096), (300, 4100),
         (300, 8185), (700, 8192), (8300, 520), (9000, 96), (8200, 2041)]


@pytest.mark.parametrize("center", [True, False], ids=["centred", "rms"])
@pytest.mark.parametrize("shape", TURNS, ids=lambda s: "x".join(map(str, s)))
def test_norm_gradient_over_several_turns(shape, center):
    rows, cols = shape
    say("norm, several turns", shape, center)
    for seed, (xt, rt, wt, dt) in enumerate([("bf16", "bf16", "bf16", "bf16"), ("bf16", "f32", "f32", "f32"), ("f32", None, "f32", "bf16")]):
        x, d = draw(rows, cols, seed, xt), draw(rows, cols, seed + 10, dt)
        r, more = (draw(rows, cols, seed + s, rt) if rt else None for s in (20, 30))
        w = (1 + 0.2 * draw(1, cols, seed + 40, "f32")[0]).to(T[wt])
        b = draw(1, cols, seed + 50, wt)[0] if center else None
        against_formula(x, w, b, r, d, more, center)


@pytest.mark.parametrize("shape", [(3, 8), (700, 136), (600, 1501), (600, 2048), (1200, 520), (300, 8192), (3, 8200), (5, 3)],
                         ids=lambda s: "x".join(map(str, s)))
def test_a_sum_s_gradient_of_another_type_than_the_sum(shape):
    rows, cols = shape
    say("norm, d_total of another type", shape)
    for seed, (rt, mt) in enumerate([("f32", "bf16"), ("bf16", "f32")]):
        x, r, d = draw(rows, cols, seed, "bf16"), draw(rows, cols, seed + 1, rt), draw(rows, cols, seed + 2, "bf16")
        w, b = (draw(1, cols, seed + s, "bf16")[0] for s in (3, 4))
        against_formula(x, w, b, r, d, draw(rows, cols, seed + 5, mt), True)


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(5, 72), (5, 1501), (5, 40001), (2500, 520), (1777, 1501), (600, 4096), (300, 8185)],
                         ids=lambda s: "x".join(map(str, s)))
def test_the_norm_s_gradient_may_take_its_operands_places(shape, t):
    """In the C call: d_x where d_out was and where d_total was, over one turn and several."""
    from test_train_cpu import call, m

    rows, cols = shape
    say("norm, in place", shape, t)
    code = {"f32": 0, "bf16": 1}[t]
    at = lambda v: m(*(v.shape if v.dim() == 2 else (1, *v.shape)), code, data=v.data_ptr())  # noqa: E731
    p = lambda v: ctypes.c_void_p(v.data_ptr())  # noqa: E731
    x, r, d, more = (draw(rows, cols, s, t) for s in range(4))
    w = draw(1, cols, 5, t)[0]
    n = wb.add_layer_norm(x, w, None, r)
    want = wb.add_layer_norm_backward(d, n, w, d_total=more)
    size = ctypes.c_size_t(0)
    assert call("wb_add_layer_norm_backward_workspace", ctypes.c_int64(rows), ctypes.c_int64(cols), ctypes.byref(size)) == 0
    ws = torch.empty(size.value, dtype=torch.uint8, device="cuda")
    for place in (0, 1):
        ops = [d.clone(), more.clone()]
        dw = torch.empty_like(w)
        assert call("wb_add_layer_norm_backward", at(ops[0]), at(n.total), at(w), at(ops[1]), p(n.mean), p(n.inv), at(ops[place]), None,
                    at(dw), None, p(ws), size, None) == 0
        assert torch.equal(ops[place], want.x) and torch.equal(dw, want.weight)
        assert torch.equal(ops[1 - place], (d, more)[1 - place])


# ---- past the caches: more than 128 MB a launch, and rows off the 16-byte grid ---------------------


@pytest.mark.parametrize("center", [True, False], ids=["centred", "rms"])
@pytest.mark.parametrize("cols", [1501, 4099, 8195])
def test_norm_past_the_caches(cols, center):
    rows = 20_000_000 // cols
    say("norm, large", rows, cols, center)
    x, r, d, more = (draw(rows, cols, s, "bf16") for s in range(4))
    w, b = (draw(1, cols, s, "bf16")[0] for s in (4, 5))
    n, got = against_formula(x, w, b, r, d, more, center)
    # a row is the same in a launch that stays in the caches
    for lo in (0, rows // 2, rows - 7):
        part = slice(lo, lo + 7)
        few = wb.add_layer_norm(x[part], w, b, r[part], eps=1e-3, center=center)
        assert torch.equal(few.out, n.out[part]) and torch.equal(few.inv, n.inv[part])
        assert torch.equal(wb.add_layer_norm_backward(d[part], few, w, d_total=more[part]).x, got.x[part])


@pytest.mark.parametrize("kind,gated,keep", [("silu", True, True), ("gelu", True, False), ("silu", False, True), ("none", True, True)])
@pytest.mark.parametrize("cols", [1501, 4099])
def test_activation_past_the_caches(cols, kind, gated, keep):
    rows = 36_000_000 // cols
    say("activation, large", rows, cols, kind, gated, keep)
    x, d = draw(rows, cols * (2 if gated else 1), 1, "bf16") * 2, draw(rows, cols, 2, "bf16")
    a = wb.activate(x, kind, gated=gated, checkpoint=keep)
    got = wb.activate_backward(d, a)
    for lo in (0, rows // 3, rows - 5):
        part = slice(lo, lo + 5)
        few = wb.activate(x[part], kind, gated=gated, checkpoint=keep)
        assert torch.equal(few.out, a.out[part])
        assert torch.equal(wb.activate_backward(d[part], few), got[part])
        ref.check(a.out[part], *tr.activate(x[part].cpu(), kind, gated), "activation")
        z, off = x[part].double().cpu(), 0.0
        if keep:
            codes, scales = tr.kept(x[part].cpu(), gated)
            assert torch.equal(a.saved[part].view(torch.uint8).cpu(), codes.view(torch.uint8))
            assert torch.equal(a.scales[part].cpu(), scales)
            z, off = tr.kept_values(codes, scales, gated), ref.U32
        ref.check(got[part], *tr.activate_backward(d[part].cpu(), z, kind, gated, off), "gradient")
    # all of it in launches that stay in the caches
    step = rows // 9 + 1
    for lo in range(0, rows, step):
        part = slice(lo, lo + step)
        few = wb.activate(x[part], kind, gated=gated, checkpoint=keep)
        assert torch.equal(few.out, a.out[part]) and torch.equal(wb.activate_backward(d[part], few), got[part])
        if keep:
            assert torch.equal(few.saved.view(torch.uint8), a.saved[part].view(torch.uint8)) and torch.equal(few.scales, a.scales[part])


@pytest.mark.parametrize("cols", [203, 1501, 4099])
def test_dispatch_and_collect_past_the_caches(cols):
    k = 4
    rows = 80_000_000 // (cols * k)
    say("dispatch, large", rows, cols)
    z = draw(rows, 8, 1, "f32")
    mask = torch.rand(rows, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda") > 0.1
    r = wb.route(z, k, mask=mask)
    x, d, y = draw(rows, cols, 3, "bf16"), draw(rows, cols, 4, "bf16"), draw(rows * k, cols, 5, "bf16")
    there, at = r.positions >= 0, r.positions.long().clamp(min=0)
    assert torch.equal(wb.dispatch(x, r), torch.where(r.tokens[:, None] >= 0, x[r.tokens.long().clamp(min=0)], 0))
    out, dx = wb.collect(y, r, residual=x), wb.dispatch_backward(y, r)
    d_y, d_g = wb.collect_backward(d, y, r)
    by_place = torch.zeros(rows * k, device="cuda")
    by_place[at[there]] = r.gates[there]
    assert torch.equal(d_y, torch.where(r.tokens[:, None] >= 0, (d[r.tokens.long().clamp(min=0)].float() * by_place[:, None]).bfloat16(), 0))
    for part in torch.arange(rows, device="cuda").split(1 + 8_000_000 // (cols * k)):
        v = y[at[part]].double() * there[part][..., None]
        g = r.gates[part].double()[..., None]
        terms = v * d[part].double()[:, None]
        for got, want, err in ((out[part], (v * g).sum(1) + x[part].double(), ((v * g).abs().sum(1) + x[part].double().abs()) * ref.U32 * (k + 1)),
                               (dx[part], v.sum(1), v.abs().sum(1) * ref.U32 * k),
                               (d_g[part], terms.sum(2), terms.abs().sum(2) * ref.U32 * tr.depth(cols))):
            ref.check(got, want.cpu(), err.cpu(), "large")


@pytest.mark.parametrize("cols,count,vocab", [(1501, 25000, 30000), (203, 340000, 5), (4099, 300, 17000)])
def test_embedding_past_the_caches(cols, count, vocab):
    say("embedding, large", cols, count, vocab)
    g = torch.Generator().manual_seed(1)
    tokens = (torch.rand(count, generator=g, dtype=torch.float64) * math.log(vocab + 1)).exp().long().clamp(max=vocab) - 1
    w, d = draw(vocab, cols, 2, "bf16"), draw(count, cols, 3, "bf16")
    got = wb.embedding(tokens.cuda(), w, scale=1.5)
    assert torch.equal(got, (w[tokens.cuda()].float() * 1.5).bfloat16())
    back = wb.embedding_backward(d, tokens.cuda(), vocab, scale=1.5)
    ref.check(back, *tr.embedding_backward(d.cpu(), tokens, vocab, 1.5, 0), "gradient")
