"""Every tile of the products against the formula in 64 bits: each type of
operand, each way of the rows (straight to LDS, by way of registers), plain and
stacked, with the epilogues that a tile forms in its own way. Which size takes
which tile is ops_tiles' to say; test_ops_cpu.py holds that against the library."""

import pytest
import torch

import ops_ref as ref
import ops_tiles as tiles
import paper_2609_25442_amd as wb
from gpu_util import say

pytestmark = pytest.mark.gpu
CASES = [(key, size) for key, sizes in tiles.SIZES.items() for size in sizes]


def operands(g, f8, rows, k):
    """Rows as they are given, and their scales (of rows: the caller repeats them for a weight's blocks)."""
    v = torch.randn(rows, k, generator=g, device="cuda")
    return (v * 100).clamp(-448, 448).to(torch.float8_e4m3fn) if f8 else v.bfloat16()


def scales(g, rows, k, like):
    return torch.rand(rows, ref.blocks(k), generator=g, device="cuda").add_(0.5).mul_(like)


@pytest.mark.parametrize("key,size", CASES, ids=lambda v: "-".join(map(str, v)).replace("True", "f8").replace("False", "bf16"))
def test_product(key, size):
    say("tile", key, size)
    f8, (form, rows, n, k, experts) = key[1], size
    form = tiles.FORMS[form]
    assert tiles.form_of_size(f8, size)[:2] == (key[0], key[2])
    g = torch.Generator(device="cuda").manual_seed(rows + n + k)
    gated, cols = form.get("gated", False), n // 2 if form.get("gated") else n
    gather = experts > 0 and key[2] == "direct"
    x = operands(g, f8, rows // 2 + 1 if gather else rows, k)
    w = [operands(g, f8, n, k) for _ in range(max(1, experts))]
    if not f8:
        w = [(m.float() * k ** -0.5).bfloat16() for m in w]
    xs = scales(g, x.shape[0], k, 0.01) if f8 else None
    ws = [scales(g, ref.blocks(n), k, 0.01 * k ** -0.5) for _ in w] if f8 else None
    b = [torch.randn(n, generator=g, device="cuda") for _ in w] if form.get("bias") else None
    r = torch.randn(rows, cols, generator=g, device="cuda").bfloat16() if form.get("residual") else None
    more = dict(x_scales=xs, activation=form.get("activation", "none"), gated=gated, residual=r, out_dtype=form["out"])
    if not experts:
        parts = [(slice(0, rows), slice(0, rows), 0)]
        got = wb.linear(x, w[0], b and b[0], weight_scales=ws and ws[0], **more)
    else:
        # uneven, some without rows, the last row the last expert's
        cut = torch.sort(torch.randint(0, rows + 1, (experts - 1,), generator=torch.Generator().manual_seed(k)))[0].tolist()
        at = [0, *cut, rows]
        at[2] = at[1]
        tokens = torch.randint(0, x.shape[0], (rows,), generator=g, device="cuda", dtype=torch.int32) if gather else None
        parts = [(slice(at[e], at[e + 1]), tokens[at[e]:at[e + 1]].long() if gather else slice(at[e], at[e + 1]), e)
                 for e in range(experts)]
        got = wb.expert_linear(x, torch.stack(w), torch.tensor(at, dtype=torch.int32, device="cuda"), tokens,
                               torch.stack(b) if b else None, weight_scales=torch.stack(ws) if f8 else None, **more)
    want, err = [], []
    for mine, source, e in parts:
        o, d = ref.product(x[source], w[e], b and b[e], more["activation"], gated, None if r is None else r[mine],
                           None if xs is None else xs[source], ws and ws[e])
        want.append(o.cpu())
        err.append(d.cpu())
    want, err = torch.cat(want), torch.cat(err)
    if form["out"] == "f8e4m3":
        ref.check_f8(got[0], got[1], want, err, "product")
    else:
        assert got.dtype == ref.TORCH[form["out"]]
        ref.check(got, want, err, "product")
