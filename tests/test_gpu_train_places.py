"""dispatch and its gradient, and collect's, over integers that no router wrote:
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
        x, d = (ref.randn(rows, cols, seed=s, dtype=t) for s in (1, 2))
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
    d_y, d_g = wb.collect_backward(x, y, r)
    assert d_y[:, 0].tolist() == [5, 2, 7, 0] and d_g.tolist() == [[16, 0, 16], [16, 0, 0]]
