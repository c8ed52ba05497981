"""One MoE layer on the tensors that unpacking leaves on a rollout rank.

Moves a small DeepSeek-V3-shaped model from its trainer layout into a rollout
rank's fp8 tensors (pack, stand-in network, unpack), then runs a layer on them:
residual norm, router, experts' products, shared expert, weighted sum; and one
router step of the trainer: its balance loss and the gradient. Run from the
repository's root on a GPU:

    python examples/moe_layer.py [tokens]
"""

from __future__ import annotations

import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

import paper_2609_25442_amd as wb  # noqa: E402
import synthetic_checkpoint as sc  # noqa: E402
from synthetic_checkpoint.workloads import scaled  # noqa: E402


def update(workload: dict) -> tuple[wb.Layout, list]:
    """The rollout rank's layout and its tensors after one transfer."""
    tr, ro = (wb.Layout.describe(workload["model"], workload[side]) for side in ("trainer", "rollout"))
    shapes = tr.tensors()
    rank = workload["unpack_rank"]
    plan = wb.Plan(tr, ro, wb.RECEIVER, rank)
    plan.upload(torch.empty(max(256, plan.workspace_bytes), dtype=torch.uint8, device="cuda"))
    recv = torch.zeros(plan.buffer_bytes, dtype=torch.uint8, device="cuda")
    values = {}
    for sender in range(tr.nranks):
        held = [torch.zeros(lc["numel"], dtype=wb.torch_dtype(lc["dtype"]), device="cuda") for lc in tr.locals(sender)]
        for t, r0, r1, c0, c1, u, base, ld, transposed in tr.placements(sender):
            if t not in values:
                rows, cols = shapes[t][1:]
                values[t] = sc.values_torch(t, rows, cols, "bf16", "cuda")
            block = values[t][r0:r1, c0:c1]
            block = block.t() if transposed else block
            held[u].as_strided(block.shape, (ld, 1), base).copy_(block)
        p = wb.Plan(tr, ro, wb.SENDER, sender)
        p.upload(torch.empty(max(256, p.workspace_bytes), dtype=torch.uint8, device="cuda"))
        send = torch.empty(max(1, p.buffer_bytes), dtype=torch.uint8, device="cuda")
        p.pack(held, send)
        at, to, n = plan.region(sender, rank)
        recv[to:to + n] = send[at:at + n]
    tensors = wb.allocate_locals(ro, rank)
    plan.unpack(recv, tensors)
    return ro, tensors


def layer(x, residual, norm_weight, w: dict, k: int, first: int) -> dict:
    """One layer on the rank whose experts are first, first + 1, ... The rest
    of a token's experts are other ranks'; their sums are added over ranks."""
    local = w["experts.w13"].shape[0]
    h, _, total = wb.add_rms_norm(x, norm_weight, residual)
    q, q_scales, _ = wb.add_rms_norm(total, norm_weight, out_dtype="f8e4m3")
    logits = wb.linear(h, w["router"], out_dtype="f32")
    r = wb.route(logits, k)
    mine = r.offsets[first:first + local + 1]
    act, act_scales = wb.expert_linear(q, w["experts.w13"], mine, tokens=r.tokens, x_scales=q_scales,
                                       weight_scales=w["experts.w13_scale"], activation="silu", gated=True,
                                       out_dtype="f8e4m3")
    y = wb.expert_linear(act, w["experts.w2"], mine, x_scales=act_scales, weight_scales=w["experts.w2_scale"])
    shared, shared_scales = wb.linear(q, w["shared.w13"], x_scales=q_scales, weight_scales=w["shared.w13_scale"],
                                      activation="silu", gated=True, out_dtype="f8e4m3")
    base = wb.linear(shared, w["shared.w2"], x_scales=shared_scales, weight_scales=w["shared.w2_scale"], residual=total)
    out = wb.combine(y, r.positions, r.gates, residual=base, span=mine)
    return dict(h=h, total=total, q=q, q_scales=q_scales, logits=logits, routing=r, mine=mine, act=act,
                act_scales=act_scales, y=y, shared=shared, shared_scales=shared_scales, base=base, out=out)


def router_step(x, router, k: int):
    """(balance loss, gradient of the router's weight) of a batch, as the
    trainer takes it: the gates go on into the experts, here into their sum of
    squares."""
    router = router.detach().float().requires_grad_()
    r = wb.route(x.float() @ router.t(), k)
    (r.loss + r.gates.square().mean()).backward()
    return r.loss.detach(), router.grad


def main(tokens: int = 64, name: str = "dsv3_ep64_to_ep8_fp8", k: int = 4) -> dict:
    workload = scaled(name)
    layout, tensors = update(workload)
    rank = workload["unpack_rank"]
    w = {lc["name"][len("layers.0."):]: t for lc, t in zip(layout.locals(rank), tensors) if lc["name"].startswith("layers.0.")}
    hidden = workload["model"]["hidden"]
    g = torch.Generator(device="cuda").manual_seed(0)
    x, residual = (torch.randn(tokens, hidden, generator=g, device="cuda").bfloat16() for _ in range(2))
    norm_weight = torch.ones(hidden, dtype=torch.bfloat16, device="cuda")
    first = rank * w["experts.w13"].shape[0]
    got = layer(x, residual, norm_weight, w, k, first)
    loss, grad = router_step(got["h"], w["router"], k)
    return dict(got, x=x, residual=residual, norm_weight=norm_weight, weights=w, first=first, k=k, loss=loss, grad=grad)


if __name__ == "__main__":
    got = main(int(sys.argv[1]) if len(sys.argv) > 1 else 64)
    r = got["routing"]
    torch.cuda.synchronize()
    print(f"{got['out'].shape[0]} tokens: {int(got['mine'][-1] - got['mine'][0])} of {int(r.offsets[-1])} expert rows on this rank, "
          f"output rms {float(got['out'].float().square().mean().sqrt()):.4f}, balance loss {float(got['loss']):.4f}, "
          f"gradient norm {float(got['grad'].norm()):.3g}")
