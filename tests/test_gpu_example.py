"""The example runs a transfer and a layer on what it unpacked: every step's
result against its formula in 64 bits, from the results before it."""

import importlib.util
import os

import pytest
import torch

import ops_ref as ref
from gpu_util import say

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("moe_layer", os.path.join(ROOT, "examples", "moe_layer.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


@pytest.mark.parametrize("tokens", [1, 50])
def test_the_example_layer(tokens):
    say("example", tokens)
    got = example().main(tokens)
    torch.cuda.synchronize()
    r, w = got["routing"], {n: t.cpu() for n, t in got["weights"].items()}
    c = {n: t.cpu() for n, t in got.items() if isinstance(t, torch.Tensor)}
    want, err, total, total_err = ref.norm(c["x"], c["norm_weight"], c["residual"], 1e-6)
    ref.check(c["h"], want, err, "norm")
    ref.check(c["total"], total, total_err, "total")
    want, err, _, _ = ref.norm(c["total"], c["norm_weight"], None, 1e-6)
    ref.check_f8(c["q"], c["q_scales"], want, err, "fp8 norm")
    ref.check(c["logits"], *ref.product(c["h"], w["router"], None, "none", False, None), "logits")
    want = ref.route(c["logits"], got["k"], None, True)
    for f in ("experts", "positions", "tokens", "offsets"):
        assert torch.equal(getattr(r, f).cpu().long(), want[f]), f
    lo, at = int(c["mine"][0]), c["mine"].tolist()
    act, act_err, y, y_err = [], [], [], []
    for e in range(len(at) - 1):
        rows = slice(at[e], at[e + 1])
        a, b = ref.product(c["q"][want["tokens"][rows]], w["experts.w13"][e], None, "silu", True, None,
                           c["q_scales"][want["tokens"][rows]], w["experts.w13_scale"][e])
        act.append(a), act_err.append(b)
        a, b = ref.product(c["act"][rows], w["experts.w2"][e], None, "none", False, None, c["act_scales"][rows],
                           w["experts.w2_scale"][e])
        y.append(a), y_err.append(b)
    if at[-1] > lo:
        ref.check_f8(c["act"][lo:at[-1]], c["act_scales"][lo:at[-1]], torch.cat(act), torch.cat(act_err), "experts' first product")
        ref.check(c["y"][lo:at[-1]], torch.cat(y), torch.cat(y_err), "experts' second product")
    a, b = ref.product(c["q"], w["shared.w13"], None, "silu", True, None, c["q_scales"], w["shared.w13_scale"])
    ref.check_f8(c["shared"], c["shared_scales"], a, b, "shared expert's first product")
    a, b = ref.product(c["shared"], w["shared.w2"], None, "none", False, c["total"], c["shared_scales"], w["shared.w2_scale"])
    ref.check(c["base"], a, b, "shared expert's second product")
    pos, gates = want["positions"], r.gates.cpu().double()
    there = ((pos >= lo) & (pos < at[-1])).double()
    rows_of = torch.nan_to_num(c["y"].double())[pos.clamp(min=0)] * (there * gates)[..., None]
    out = rows_of.sum(1) + c["base"].double()
    ref.check(c["out"], out, (rows_of.abs().sum(1) * 6 + out.abs()) * ref.U32, "sum")
    assert torch.isfinite(got["grad"]).all() and float(got["loss"]) > 0
