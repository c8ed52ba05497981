"""dispatch and collect, there and back, over integers that no router wrote:
places outside the rows, of other rows, and named twice. A choice counts where
its place is one of the call's, says its row, and no earlier choice of the row
has it; the operators and their gradients agree on that."""

import pytest
import torch

import ops_ref as ref
import paper_2609_25442_amd as wb
from gpu_util import say

pytestmark = pytest.mark.gpu
U32 = ref.U32


def counts(positions, tokens, span):
    """Whether each choice counts, from the rule above."""
    rows, k = positions.shape
    lo, hi = (0, len(tokens)) if span is None else (max(0, span[0]), min(span[1], len(tokens)))
    on = torch.zeros(rows, k, dtype=torch.bool)
    for t in range(rows):
        for i in range(k):
            p = int(positions[t, i])
            on[t, i] = lo <= p < hi and int(tokens[p]) == t and p not in positions[t, :i].tolist()
    return on


def any_routing(rows, k, places, seed):
    """Places that mostly name their row, some taken by others, some twice in a row, some that are none."""
    g = torch.Generator().manual_seed(seed)
    tokens = torch.randint(-1, rows + 1, (places,), generator=g)
    positions = torch.randint(-3, places + 3, (rows, k), generator=g)
    for t in range(rows):
        mine = torch.nonzero(tokens == t)[:, 0]
        for i in range(k):
            if len(mine) and torch.rand((), generator=g) < 0.7:
                positions[t, i] = mine[torch.randint(0, len(mine), (), generator=g)]  # now and then the same again
    return positions, tokens


def of(positions, tokens, gates):
    e = torch.zeros(1, dtype=torch.int32, device="cuda")
    return wb.Routing(e, gates.cuda(), positions.int().cuda(), tokens.int().cuda(), e, e, e, e, None, True)


@pytest.mark.parametrize("shape", [(1, 1, 1, 8), (1, 2, 3, 40), (5, 2, 10, 7), (20, 3, 60, 72), (33, 8, 264, 129), (9, 64, 300, 64),
                                   (3, 64, 20, 4099), (40, 5, 100, 2049), (6, 4, 24, 20001), (70, 2, 1, 264), (4, 2, 0, 16)],
                         ids=lambda s: "x".join(map(str, s)))
def test_operators_and_gradients_agree_on_what_counts(shape):
    rows, k, places, cols = shape
    say("places", shape)
    positions, tokens = any_routing(rows, k, places, 1)
    for t, span in (("f32", None), ("bf16", None), ("f32", [places // 4, places - places // 3])):
        on = counts(positions, tokens, span)
        where = None if span is None else torch.tensor(span, dtype=torch.int32, device="cuda")
        x, d, res = (ref.randn(rows, cols, seed=s, dtype=t) for s in (1, 2, 3))
        y = ref.randn(places, cols, seed=4, dtype=t)
        gates = ref.randn(rows, k, seed=5)
        r = of(positions, tokens, gates)
        row, i = torch.nonzero(on, as_tuple=True)
        at = positions[row, i]
        want = torch.zeros(places, cols, dtype=x.dtype)
        want[at] = x[row]
        assert torch.equal(wb.dispatch(x.cuda(), r, span=where).cpu(), want)
        dx, size = torch.zeros(rows, cols).double(), torch.zeros(rows, cols).double()
        dx.index_add_(0, row, y.double()[at])
        size.index_add_(0, row, y.double()[at].abs())
        ref.check(wb.dispatch_backward(y.cuda(), r, span=where), dx, size * U32 * k, "dispatch's gradient")
        g = gates.double()[row, i][:, None]
        out, size = res.double(), res.double().abs()
        out.index_add_(0, row, g * y.double()[at])
        size.index_add_(0, row, (g * y.double()[at]).abs())
        ref.check(wb.collect(y.cuda(), r, residual=res.cuda(), span=where), out, size * U32 * (k + 1), "collect")
        d_y, d_g = wb.collect_backward(d.cuda(), y.cuda(), r, span=where)
        of_y, of_g, e_g = torch.zeros(places, cols).double(), torch.zeros(rows, k).double(), torch.zeros(rows, k).double()
        of_y[at] = g * d.double()[row]
        terms = d.double()[row] * y.double()[at]
        of_g[row, i], e_g[row, i] = terms.sum(1), terms.abs().sum(1) * U32 * (128 + cols // 256)
        ref.check(d_y, of_y, of_y.abs() * U32, "gradient of y")
        ref.check(d_g, of_g, e_g, "gradient of the gates")


def test_a_place_named_twice_in_a_row_is_the_first_choice_s():
    positions, tokens = torch.tensor([[1, 1, 0], [2, 0, 2]]), torch.tensor([0, 0, 1, -1])
    gates = torch.tensor([[2.0, 3.0, 5.0], [7.0, 11.0, 13.0]])
    r = of(positions, tokens, gates)
    x, y = torch.ones(2, 16, device="cuda"), torch.ones(4, 16, device="cuda")
    assert wb.dispatch(x, r)[:, 0].tolist() == [1, 1, 1, 0]
    assert wb.dispatch_backward(y, r)[:, 0].tolist() == [2, 1]
    assert wb.collect(y, r)[:, 0].tolist() == [7, 7]
    d_y, d_g = wb.collect_backward(x, y, r)
    assert d_y[:, 0].tolist() == [5, 2, 7, 0] and d_g.tolist() == [[16, 0, 16], [16, 0, 0]]


def test_collect_of_places_that_say_another_row():
    """An edited routing: a place that tokens no longer gives to a row adds nothing, as its gradients are zeros."""
    z = ref.randn(12, 6, seed=1).cuda()
    r = wb.route(z, 2)
    gone = r.positions[3, 1].item()
    tokens = r.tokens.clone()
    tokens[gone] = -1
    edited = r._replace(tokens=tokens)
    y = ref.randn(24, 40, seed=2).cuda()
    y[gone] = float("nan")
    gates = r.gates.clone().requires_grad_()
    rows = y.clone().requires_grad_()
    out = wb.collect(rows, edited, gates=gates)
    assert torch.isfinite(out).all()
    out.sum().backward()
    assert gates.grad[3, 1] == 0 and torch.isfinite(gates.grad).all() and not rows.grad[gone].any()
    other = torch.arange(12, device="cuda") != 3
    assert torch.equal(out[other], wb.combine(y, r.positions, r.gates)[other])


def test_collect_refuses_what_is_no_tensor():
    r = of(torch.zeros(2, 1).long(), torch.zeros(2).long(), torch.ones(2, 1))
    x = torch.ones(2, 8, device="cuda")
    for call in (lambda: wb.collect(None, r), lambda: wb.collect([1.0], r), lambda: wb.collect(x[0], r), lambda: wb.collect(x[:1], r),
                 lambda: wb.collect(None, r, gates=torch.ones(2, 1, device="cuda", requires_grad=True)),
                 lambda: wb.collect(x, r._replace(tokens=r.tokens.long())), lambda: wb.collect(x, r, span=r.tokens.long()),
                 lambda: wb.collect(x, r, out_dtype="f8e4m3"), lambda: wb.collect(x.half(), r), lambda: wb.collect(x, r, residual=x[:1])):
        with pytest.raises(wb.WbError):
            call()


def test_collect_into_the_residual_s_place_and_of_rows_that_start_anywhere():
    import ctypes

    from test_train_cpu import call, m

    r = wb.route(ref.randn(30, 8, seed=1).cuda(), 3)
    p = lambda v: ctypes.c_void_p(v.data_ptr())  # noqa: E731
    for cols in (72, 1501, 4099):
        y, res = ref.randn(90, cols, seed=2), ref.randn(30, cols, seed=3)
        want = wb.collect(y.cuda(), r, residual=res.cuda())
        assert torch.equal(want, wb.combine(y.cuda(), r.positions, r.gates, residual=res.cuda()))
        for pad, skip in ((0, 1), (3, 0), (5, 3)):
            assert torch.equal(wb.collect(ref.strided(y, pad, skip), r, residual=ref.strided(res, pad, skip)), want)
        here, rows = res.cuda(), y.cuda()
        at = lambda v: m(*v.shape, 0, data=v.data_ptr())  # noqa: E731
        assert call("wb_collect", at(rows), p(r.positions), p(r.tokens), p(r.gates), 3, at(here), None, None, at(here), None) == 0
        assert torch.equal(here, want)


def test_what_choices_that_do_not_count_hold_goes_nowhere():
    """Gates and rows that are not finite, at places of no one, of others, and named again."""
    nan, inf = float("nan"), float("inf")
    positions = torch.tensor([[0, 0, 9, -4], [1, 3, 2, 2]])
    tokens = torch.tensor([0, 0, 1, -1])
    r = of(positions, tokens, torch.tensor([[2.0, nan, inf, nan], [nan, inf, 3.0, nan]]))
    for t in ("f32", "bf16"):
        for cols in (8, 13, 520, 2500):
            y = torch.tensor([1.0, nan, 5.0, inf])[:, None].repeat(1, cols).to(ref.TORCH[t]).cuda()
            assert wb.collect(y, r)[:, -1].tolist() == [2, 15] and torch.isfinite(wb.collect(y, r)).all()
            d_y, d_g = wb.collect_backward(torch.ones(2, cols, device="cuda"), y, r)
            assert d_y[:, -1].tolist() == [2, 0, 3, 0]
            assert d_g.tolist() == [[cols, 0, 0, 0], [0, 0, 5 * cols, 0]]


def test_collect_past_four_gigabytes():
    say("collect, far rows")
    rows, cols, k = 70000, 8192, 4
    r = wb.route(ref.randn(rows, 8, seed=1).cuda(), k)
    y = torch.zeros(rows * k, cols, dtype=torch.bfloat16, device="cuda")
    y[:, 8191] = (torch.arange(rows * k, device="cuda") % 251).bfloat16()
    out = wb.collect(y, r, gates=torch.ones(rows, k, device="cuda"), out_dtype="f32")
    assert torch.equal(out[:, 8191], y[:, 8191].float()[r.positions.long()].sum(1)) and not out[:, :8191].any()
