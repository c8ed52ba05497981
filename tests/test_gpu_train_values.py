"""The gradient of the layer norm where gradients or weights are not finite:
infinities and NaN go where the formula has them, whatever their column."""

import math

import pytest
import torch

import ops_ref as ref
import paper_2609_25442_amd as wb
from gpu_util import say

pytestmark = pytest.mark.gpu


def formula(d, w, h, inv, center):
    """The gradient of the sum in 64 bits, step by step, so that infinities meet as they do in the formula."""
    g = d.double() * w.double()
    n = d.shape[1]
    s = g - g.sum(1, keepdim=True) / n if center else g
    return (s - h * ((g * h).sum(1, keepdim=True) / n)) * inv


@pytest.mark.parametrize("center", [True, False], ids=["centred", "rms"])
@pytest.mark.parametrize("cols", [5, 8, 13, 264, 520, 1000, 1501, 2048, 4096, 4100, 7168, 8185, 8200])
def test_layer_norm_gradient_of_infinite_and_nan_gradients(cols, center):
    say("norm gradient, not finite", cols, center)
    rows = 9
    for seed, (t, dt) in enumerate([("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")]):
        x, w = ref.randn(rows, cols, seed=seed, dtype=t).cuda(), ref.randn(cols, seed=seed + 10, dtype=t).cuda()
        clean = ref.randn(rows, cols, seed=seed + 20, dtype=dt).cuda()
        n = wb.add_layer_norm(x, w, w, center=center)
        mean = n.mean.double()[:, None] if center else 0.0
        h = (x.double() - mean) * n.inv.double()[:, None]
        d = clean.clone()
        d[1, cols - 1], d[2, max(0, cols - 3)], d[3, 0], d[4, cols // 2] = math.inf, -math.inf, math.inf, -math.inf
        d[5, cols - 1], d[6, max(0, cols - 8)] = math.nan, math.inf
        want = formula(d, w, h, n.inv.double()[:, None], center)
        got = wb.add_layer_norm_backward(d, n, w)
        plain = wb.add_layer_norm_backward(clean, n, w)
        bad = list(range(1, 7))
        assert torch.equal(torch.isnan(got.x[bad]), torch.isnan(want[bad])), "NaN in other places"
        there = torch.isinf(want[bad])
        assert torch.equal(got.x[bad].double()[there], want[bad][there]), "infinities"
        assert torch.equal(got.x[[0, 7, 8]], plain.x[[0, 7, 8]])
        # a column's sum is not finite where one of its own gradients is not
        hit = ~torch.isfinite(d).all(0)
        for a, b in ((got.weight, plain.weight), (got.bias, plain.bias)):
            assert not torch.isfinite(a[hit]).any() and torch.equal(a[~hit], b[~hit])


@pytest.mark.parametrize("cols", [13, 264, 1501, 7168, 8185])
def test_layer_norm_gradient_of_an_infinite_weight(cols):
    x, d = ref.randn(4, cols, seed=1).cuda(), ref.randn(4, cols, seed=2).cuda()
    for at in (0, cols - 8, cols - 1):
        w = ref.randn(cols, seed=3).cuda()
        w[at] = math.inf
        n = wb.add_layer_norm(x, w)
        h = (x.double() - n.mean.double()[:, None]) * n.inv.double()[:, None]
        want = formula(d, w, h, n.inv.double()[:, None], True)
        got = wb.add_layer_norm_backward(d, n, w)
        assert torch.equal(torch.isnan(got.x), torch.isnan(want))
        assert torch.equal(got.x.double()[torch.isinf(want)], want[torch.isinf(want)])
        assert torch.isfinite(got.weight).all()
