"""Timed cases of the operators that use a rollout rank's tensors: the residual
norm in front of a layer, the router of an MoE layer with its balance loss, the
products with plain and with stacked expert weights, and the weighted sum of a
token's expert rows.

A case names one operator (``op``) and its sizes:

* ``norm``     ``rows`` tokens of ``cols`` values, added to a residual and
               normed, out as bf16 or as fp8 with a scale per 128 values;
* ``route``    ``rows`` tokens over ``experts`` experts, ``k`` of them chosen;
               with ``step`` the gradient of the logits too;
* ``linear``   ``rows`` tokens times a weight [``n``, ``cols``];
* ``experts``  ``rows`` routed rows over ``experts`` stacked weights;
* ``combine``  ``rows`` tokens, each the sum of ``k`` expert rows.

fp8 operands are E4M3 values with fp32 scales, of 128 values of a row for
activations and of 128x128 blocks for weights, as ranks hold them.
"""

import math
import random

import torch

own = False

EPS = 1e-6
STD = 0.02  # spread of a trained weight matrix
BLOCK = 128
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "f8": torch.float8_e4m3fn}
BYTES = {"bf16": 2, "f32": 4, "f8": 1}


def listed():
    return [
        # one decode step of four sequences: the call is what costs
        dict(name="norm_decode", op="norm", rows=4, cols=7168, dtype="bf16", out="f8", residual=True),
        # a long prompt batch
        dict(name="norm_prefill", op="norm", rows=16384, cols=7168, dtype="bf16", out="f8", residual=True),
        # one decode step of 32 sequences, eight experts
        dict(name="route_decode", op="route", rows=32, experts=8, k=2, dtype="bf16", mask=False, renorm=True,
             step=False),
        # a training microbatch with padding, 256 experts: forward and gradient
        dict(name="route_train", op="route", rows=32768, experts=256, k=8, dtype="f32", mask=True, renorm=True,
             step=True),
        # fused qkv of one token
        dict(name="linear_token", op="linear", rows=1, n=6144, cols=4096, dtype="bf16", gated=False, act="none",
             bias=False, residual=False, out="bf16"),
        # gate and up of a prompt batch
        dict(name="linear_prefill", op="linear", rows=8192, n=28672, cols=4096, dtype="bf16", gated=True, act="silu",
             bias=False, residual=False, out="bf16"),
        # a model whose sizes are no multiples of anything, with everything in the epilogue
        dict(name="linear_ragged", op="linear", rows=333, n=3442, cols=1500, dtype="bf16", gated=False, act="gelu",
             bias=True, residual=True, out="bf16"),
        # down product of a shared expert, added to the layer's sum
        dict(name="linear_fp8", op="linear", rows=4096, n=7168, cols=2048, dtype="f8", gated=False, act="none",
             bias=False, residual=True, out="bf16"),
        # one decode step: 128 routed rows on a rank with 32 experts
        dict(name="experts_decode", op="experts", rows=128, experts=32, n=4096, cols=7168, dtype="f8", gated=True,
             act="silu", bias=False, residual=False, out="f8", gather=True),
        # the same rank with a prompt batch
        dict(name="experts_prefill", op="experts", rows=8192, experts=32, n=4096, cols=7168, dtype="f8", gated=True,
             act="silu", bias=False, residual=False, out="f8", gather=True),
        # the sums of a small decode step
        dict(name="combine_decode", op="combine", rows=16, cols=4096, k=2, dtype="bf16", residual=True),
        # the sums of a prompt batch
        dict(name="combine_prefill", op="combine", rows=4096, cols=7168, k=8, dtype="bf16", residual=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A length of the range: as drawn in a third of the cases, else a multiple of 64."""
    n = _log(rng, lo, hi)
    return n if rng.random() < 0.35 else max(64, n // 64 * 64)


def draw(rng):
    """A case of the same kinds: one to tens of thousands of rows, narrow to wide, plain and odd sizes."""
    most = max(_cost(c) for c in listed())
    while True:
        op = rng.choice(["norm", "route", "linear", "linear", "experts", "experts", "combine"])
        if op == "norm":
            c = dict(op=op, rows=_log(rng, 1, 16384), cols=_size(rng, 64, 8192), dtype=rng.choice(["bf16", "bf16", "f32"]),
                     out=rng.choice(["bf16", "f8", "f8"]), residual=rng.random() < 0.7)
        elif op == "route":
            experts = rng.choice([8, 16, 64, 256, _log(rng, 2, 512)])
            c = dict(op=op, rows=_log(rng, 1, 32768), experts=experts, k=rng.randint(1, min(8, experts)),
                     dtype=rng.choice(["bf16", "f32"]), mask=rng.random() < 0.5, renorm=rng.random() < 0.7,
                     step=rng.random() < 0.6)
        elif op == "combine":
            c = dict(op=op, rows=_log(rng, 1, 8192), cols=_size(rng, 64, 8192), k=rng.randint(1, 8),
                     dtype=rng.choice(["bf16", "bf16", "f32"]), residual=rng.random() < 0.7)
        else:
            gated = rng.random() < 0.5
            half = _size(rng, 64, 14336 if op == "linear" else 4096)
            c = dict(op=op, rows=_log(rng, 1, 8192), n=2 * half if gated else half, cols=_size(rng, 64, 8192),
                     dtype=rng.choice(["bf16", "f8"]), gated=gated, act=rng.choice(["silu", "gelu"] if gated else ["none", "none", "silu", "gelu"]),
                     bias=rng.random() < 0.3, residual=rng.random() < 0.3,
                     out=rng.choice(["bf16", "bf16", "f32", "f8"]))
            if op == "experts":
                c.update(experts=_log(rng, 1, 64), gather=rng.random() < 0.5)
        # 3072 is a width of none of this repository's models
        if _cost(c) <= most and work(c)["bytes"] <= 2e9 and 3072 not in c.values():
            return c


def _cost(c):
    w = work(c)
    return max(w["bytes"] / 5e12, w["flops"] / 5e14)


def _counts(c):
    """How many rows each expert gets, the same for every seed: uneven, as routers leave them."""
    r = random.Random(c["rows"] * 1009 + c["experts"])
    share = [math.exp(r.gauss(0.0, 0.7)) for _ in range(c["experts"])]
    got, left, total = [], c["rows"], sum(share)
    for s in share:
        n = min(left, int(round(left * s / total)) if total > 0 else left)
        got.append(n)
        left, total = left - n, total - s
    got[-1] += left
    return got


def _columns(c):
    return c["n"] // 2 if c["gated"] else c["n"]


def work(c):
    rows = c["rows"]
    if c["op"] == "norm":
        n, es = rows * c["cols"], BYTES[c["dtype"]]
        out = n * BYTES[c["out"]] + (4 * rows * -(-c["cols"] // BLOCK) if c["out"] == "f8" else 0)
        return {"bytes": n * es * (3 if c["residual"] else 1) + out + c["cols"] * 2, "flops": 6 * n}
    if c["op"] == "route":
        n, es = rows * c["experts"], BYTES[c["dtype"]]
        there = n * es + rows * (1 if c["mask"] else 0) + 16 * rows * c["k"] + 8 * c["experts"]
        back = 2 * n * es + rows * (1 if c["mask"] else 0) + 12 * rows * c["k"] + 4 * c["experts"]
        return {"bytes": there + (back if c["step"] else 0), "flops": n * (16 if c["step"] else 8)}
    if c["op"] == "combine":
        n, es = rows * c["cols"], BYTES[c["dtype"]]
        return {"bytes": n * es * (c["k"] + 1 + c["residual"]) + 8 * rows * c["k"], "flops": 2 * n * c["k"]}
    es, n, k = BYTES[c["dtype"]], c["n"], c["cols"]
    weights, x_rows = 1, rows
    if c["op"] == "experts":
        weights, x_rows = sum(x > 0 for x in _counts(c)), _x_rows(c)
    out = rows * _columns(c) * (BYTES[c["out"]] + (BYTES["f32" if c["out"] == "f32" else "bf16"] if c["residual"] else 0))
    scales = 0
    if c["dtype"] == "f8":
        scales += 4 * -(-k // BLOCK) * (x_rows + weights * -(-n // BLOCK))
    if c["out"] == "f8":
        scales += 4 * rows * -(-_columns(c) // BLOCK)
    return {"bytes": (x_rows * k + weights * n * k) * es + out + scales + (weights * n * 4 if c["bias"] else 0),
            "flops": 2 * rows * n * k}


def _x_rows(c):
    """Rows of x: with a gather every token sits at a few experts."""
    return max(1, c["rows"] // 4) if c["gather"] else c["rows"]


def _activations(g, rows, cols, dtype):
    """Hidden states: a few columns are much larger than the others, as in trained models."""
    x = torch.randn(rows, cols, generator=g, device="cuda")
    x.mul_(torch.rand(cols, generator=g, device="cuda").mul_(3).exp_().mul_(0.3))
    return x.to(TYPES[dtype])


def _quantised_rows(x):
    rows, cols = x.shape
    nb = -(-cols // BLOCK)
    p = torch.nn.functional.pad(x.float(), (0, nb * BLOCK - cols)).view(rows, nb, BLOCK)
    s = p.abs().amax(-1) / 448
    s = torch.where(s > 0, s, torch.ones_like(s))
    return (p / s[..., None]).view(rows, -1)[:, :cols].contiguous().to(torch.float8_e4m3fn), s


def _quantised_blocks(w):
    n, k = w.shape[-2:]
    a, b = -(-n // BLOCK), -(-k // BLOCK)
    p = torch.nn.functional.pad(w.float(), (0, b * BLOCK - k, 0, a * BLOCK - n)).view(-1, a, BLOCK, b, BLOCK)
    s = p.abs().amax((2, 4)) / 448
    s = torch.where(s > 0, s, torch.ones_like(s))
    q = (p / s[:, :, None, :, None]).view(-1, a * BLOCK, b * BLOCK)[:, :n, :k].contiguous().to(torch.float8_e4m3fn)
    return q.view(w.shape), s.view(*w.shape[:-2], a, b)


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda").manual_seed(seed)
    rows, op = c["rows"], c["op"]
    if op == "norm":
        s = dict(x=_activations(g, rows, c["cols"], c["dtype"]), residual=None,
                 weight=(1 + 0.1 * torch.randn(c["cols"], generator=g, device="cuda")).bfloat16())
        if c["residual"]:
            s["residual"] = _activations(g, rows, c["cols"], c["dtype"])
    elif op == "route":
        z = torch.randn(rows, c["experts"], generator=g, device="cuda").mul_(1.5)
        z.add_(torch.randn(c["experts"], generator=g, device="cuda").mul_(0.5))
        s = dict(logits=z.to(TYPES[c["dtype"]]), mask=None)
        if c["mask"]:
            s["mask"] = torch.rand(rows, generator=g, device="cuda") < 0.9
        if c["step"]:
            s.update(d_gates=torch.randn(rows, c["k"], generator=g, device="cuda"),
                     d_loss=torch.rand((), generator=g, device="cuda").add_(0.5).mul_(rows))
    elif op == "combine":
        k = c["k"]
        s = dict(y=_activations(g, rows * k, c["cols"], c["dtype"]), residual=None,
                 positions=torch.randperm(rows * k, generator=g, device="cuda").view(rows, k).int(),
                 gates=torch.softmax(torch.randn(rows, k, generator=g, device="cuda"), -1))
        if c["residual"]:
            s["residual"] = _activations(g, rows, c["cols"], c["dtype"])
    else:
        stack = (c["experts"],) if op == "experts" else ()
        f8 = c["dtype"] == "f8"
        x = _activations(g, _x_rows(c) if op == "experts" else rows, c["cols"], "bf16")
        w = torch.randn(*stack, c["n"], c["cols"], generator=g, device="cuda", dtype=torch.bfloat16).mul_(STD)
        s = dict(x=x, weight=w, x_scales=None, weight_scales=None, bias=None, residual=None)
        if f8:
            s["x"], s["x_scales"] = _quantised_rows(x)
            s["weight"], s["weight_scales"] = _quantised_blocks(w)
        if c["bias"]:
            s["bias"] = torch.randn(*stack, c["n"], generator=g, device="cuda")
        if c["residual"]:
            s["residual"] = _activations(g, rows, _columns(c), "f32" if c["out"] == "f32" else "bf16")
        if op == "experts":
            counts = _counts(c)
            random.Random(seed).shuffle(counts)
            at = [0]
            for n in counts:
                at.append(at[-1] + n)
            s.update(offsets=torch.tensor(at, dtype=torch.int32, device="cuda"), tokens=None, most=max(counts))
            if c["gather"]:
                s["tokens"] = torch.randint(0, x.shape[0], (rows,), generator=g, device="cuda", dtype=torch.int32)
    s["case"] = c
    return s


def run(state):
    return (_run_own if own else _run_plain)(state)


# ---- the framework's calls ---------------------------------------------------------------------


def _run_own(s):
    import paper_2609_25442_amd as wb

    c = s["case"]
    name = {"bf16": "bf16", "f32": "f32", "f8": "f8e4m3"}
    if c["op"] == "norm":
        out = c["dtype"] if c["out"] != "f8" else "f8"
        y, scales, total = wb.add_rms_norm(s["x"], s["weight"], s["residual"], eps=EPS, out_dtype=name[out])
        return [v for v in (y, scales, total) if v is not None]
    if c["op"] == "route":
        r = wb.route(s["logits"], c["k"], mask=s["mask"], renormalize=c["renorm"])
        got = [r.experts, r.gates, r.positions, r.tokens, r.counts, r.offsets, r.loss]
        if c["step"]:
            got.append(wb.route_backward(s["logits"], r, s["d_gates"], s["d_loss"]))
        return got
    if c["op"] == "combine":
        return wb.combine(s["y"], s["positions"], s["gates"], residual=s["residual"])
    more = dict(x_scales=s["x_scales"], weight_scales=s["weight_scales"], bias=s["bias"], activation=c["act"],
                gated=c["gated"], residual=s["residual"], out_dtype=name[c["out"]])
    if c["op"] == "experts":
        return wb.expert_linear(s["x"], s["weight"], s["offsets"], tokens=s["tokens"], **more)
    return wb.linear(s["x"], s["weight"], **more)


# ---- the plain forms: elementary operations in 32 bits -----------------------------------------


def _run_plain(s):
    return {"norm": _plain_norm, "route": _plain_route, "linear": _plain_linear, "experts": _plain_experts,
            "combine": _plain_combine}[s["case"]["op"]](s, s["case"])


def _rows_in_f8(y):
    """(E4M3 values, scale per 128 columns) of fp32 rows."""
    rows, cols = y.shape
    nb = -(-cols // BLOCK)
    p = torch.zeros(rows, nb * BLOCK, device=y.device)
    p[:, :cols] = y
    p = p.view(rows, nb, BLOCK)
    s = p.abs().amax(-1) / 448
    s = torch.where(s > 0, s, torch.ones_like(s))
    return (p / s[..., None]).view(rows, -1)[:, :cols].to(torch.float8_e4m3fn), s


def _plain_norm(s, c):
    t = s["x"].float()
    if s["residual"] is not None:
        t = t + s["residual"].float()
    y = t * torch.rsqrt((t * t).mean(-1, keepdim=True) + EPS) * s["weight"].float()
    got = list(_rows_in_f8(y)) if c["out"] == "f8" else [y.to(s["x"].dtype)]
    if s["residual"] is not None:
        got.append(t.to(s["residual"].dtype))
    return got


def _plain_route(s, c):
    z = s["logits"].float()
    (rows, e), k = z.shape, c["k"]
    routed = torch.ones(rows, dtype=torch.bool, device=z.device) if s["mask"] is None else s["mask"]
    top, order = torch.sort(z, dim=-1, descending=True, stable=True)
    p = torch.exp(z - top[:, :1])
    p = p / p.sum(-1, keepdim=True) * routed[:, None]
    experts = torch.where(routed[:, None], order[:, :k], -1)
    gates = p.gather(1, order[:, :k])
    if c["renorm"]:
        gates = torch.exp(top[:, :k] - top[:, :1])
        gates = gates / gates.sum(-1, keepdim=True) * routed[:, None]
    flat = torch.where(experts < 0, e, experts).view(-1)
    place = torch.sort(flat, stable=True)[1]
    counts = (flat[:, None] == torch.arange(e, device=z.device)).sum(0)
    offsets = torch.cat([counts.new_zeros(1), counts.cumsum(0)])
    here = torch.arange(rows * k, device=z.device)
    positions = torch.empty_like(place)
    positions[place] = here
    positions = torch.where(flat == e, -1, positions).view(rows, k)
    tokens = torch.where(here < offsets[-1], place // k, -1)
    n = routed.sum().clamp(min=1).float()
    share = counts.float() * (e / (k * n * n))
    loss = (share * p.sum(0)).sum()
    got = [experts.int(), gates, positions.int(), tokens.int(), counts.int(), offsets.int(), loss]
    if c["step"]:
        dp = (share * s["d_loss"]).expand(rows, e)
        dg = s["d_gates"]
        if not c["renorm"]:
            dp = dp.scatter_add(1, order[:, :k], dg)
        dz = p * (dp - (p * dp).sum(-1, keepdim=True))
        if c["renorm"]:
            dz = dz.scatter_add(1, order[:, :k], gates * (dg - (dg * gates).sum(-1, keepdim=True)))
        got.append(dz.to(s["logits"].dtype))
    return got


def _values(q, scales, per_row):
    """fp32 values of an operand."""
    if scales is None:
        return q.float()
    n, k = q.shape[-2:]
    a = scales.repeat_interleave(BLOCK, -1)[..., :k]
    return q.float() * (a if per_row else a.repeat_interleave(BLOCK, -2)[..., :n, :])


def _act(z, kind):
    if kind == "silu":
        return z / (1 + torch.exp(-z))
    if kind == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    return z


def _finish(z, s, c):
    """Activation, residual and rounding of fp32 rows."""
    if c["gated"]:
        gate, up = z.chunk(2, -1)
        a = _act(gate, c["act"]) * up
    else:
        a = _act(z, c["act"])
    if s["residual"] is not None:
        a = a + s["residual"].float()
    return list(_rows_in_f8(a)) if c["out"] == "f8" else a.to(TYPES[c["out"]])


def _plain_linear(s, c):
    z = _values(s["x"], s["x_scales"], True) @ _values(s["weight"], s["weight_scales"], False).t()
    if s["bias"] is not None:
        z = z + s["bias"]
    return _finish(z, s, c)


def _plain_experts(s, c):
    """The experts as one batched product: their rows side by side, as many as the fullest has."""
    x = _values(s["x"], s["x_scales"], True)
    here = torch.arange(c["rows"], device="cuda")
    e = torch.searchsorted(s["offsets"].long(), here, right=True) - 1
    at = here - s["offsets"].long()[e]
    rows = x[s["tokens"].long()] if s["tokens"] is not None else x
    wide = x.new_zeros(c["experts"], s["most"], c["cols"])
    wide[e, at] = rows
    z = torch.bmm(wide, _values(s["weight"], s["weight_scales"], False).transpose(1, 2).contiguous())[e, at]
    if s["bias"] is not None:
        z = z + s["bias"][e]
    return _finish(z, s, c)


def _plain_combine(s, c):
    out = (s["y"].float()[s["positions"].long()] * s["gates"][..., None]).sum(1)
    if s["residual"] is not None:
        out = out + s["residual"].float()
    return out.to(s["y"].dtype)


# ---- the definitions in 64 bits ----------------------------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "route": _exact_route, "linear": _exact_product, "experts": _exact_product,
            "combine": _exact_combine}[case["op"]](s, case)


def _scaled_exactly(y):
    """(y / s, s) with s the largest magnitude of each run of 128 columns over 448."""
    s = torch.stack([b.abs().amax(1) for b in y.split(BLOCK, 1)], 1) / 448
    s = torch.where(s > 0, s, 1.0)
    return torch.cat([b / s[:, i:i + 1] for i, b in enumerate(y.split(BLOCK, 1))], 1), s


def _exact_norm(s, c):
    t = s["x"].double() + (0 if s["residual"] is None else s["residual"].double())
    y = t / ((t.pow(2).sum(1) / c["cols"] + EPS).sqrt()[:, None]) * s["weight"].double()
    got = list(_scaled_exactly(y)) if c["out"] == "f8" else [y]
    return got + ([t] if s["residual"] is not None else [])


def _exact_route(s, c):
    z, k, e = s["logits"].double(), c["k"], c["experts"]
    on = torch.ones(c["rows"], device="cuda").double() if s["mask"] is None else s["mask"].double()
    p = torch.softmax(z, 1)
    left, chosen = z.clone(), []
    for _ in range(k):  # argmax gives no order among equals: the lowest index of the largest value
        best = (left == left.amax(1, keepdim=True)).double().argmax(1)
        chosen.append(best)
        left[torch.arange(c["rows"], device="cuda"), best] = -math.inf
    chosen = torch.stack(chosen, 1)
    pick = torch.zeros_like(z).scatter_(1, chosen, 1.0)
    gates = p.gather(1, chosen)
    if c["renorm"]:
        gates = gates / gates.sum(1, keepdim=True)
    counts, n = (pick * on[:, None]).sum(0), max(1.0, float(on.sum()))
    f = counts * e / (k * n)
    loss = (f * (p * on[:, None]).sum(0) / n).sum()
    got = [None, gates * on[:, None], None, None, None, None, loss]
    if c["step"]:
        dl, dg = s["d_loss"].double(), s["d_gates"].double()
        pg = dl / n * p * (f - (p * f).sum(1, keepdim=True))
        if c["renorm"]:
            of_gates = torch.zeros_like(z).scatter_(1, chosen, gates * (dg - (gates * dg).sum(1, keepdim=True)))
        else:
            d = torch.zeros_like(z).scatter_(1, chosen, dg)
            of_gates = p * (d - (p * d).sum(1, keepdim=True))
        got.append((pg + of_gates) * on[:, None])
    return got


def _exact_operand(q, scales, row_block):
    v = q.double()
    if scales is not None:
        i = torch.arange(v.shape[0], device="cuda") // row_block
        j = torch.arange(v.shape[1], device="cuda") // BLOCK
        v = v * scales.double()[i][:, j]
    return v


def _exact_product(s, c):
    x = _exact_operand(s["x"], s["x_scales"], 1)
    if c["op"] == "linear":
        parts = [(x, s["weight"], s["weight_scales"], s["bias"])]
    else:
        at = s["offsets"].tolist()
        if s["tokens"] is not None:
            x = x[s["tokens"].long()]
        parts = [(x[at[e]:at[e + 1]], s["weight"][e], None if s["weight_scales"] is None else s["weight_scales"][e],
                  None if s["bias"] is None else s["bias"][e]) for e in range(c["experts"]) if at[e + 1] > at[e]]
    z = torch.cat([a @ _exact_operand(w, ws, BLOCK).T + (0 if b is None else b.double()) for a, w, ws, b in parts])
    gate = z[:, :_columns(c)]
    if c["act"] == "silu":
        a = gate * torch.sigmoid(gate)
    elif c["act"] == "gelu":
        a = gate * 0.5 * torch.erfc(-gate / math.sqrt(2.0))
    else:
        a = gate
    if c["gated"]:
        a = a * z[:, _columns(c):]
    if s["residual"] is not None:
        a = a + s["residual"].double()
    return list(_scaled_exactly(a)) if c["out"] == "f8" else a


def _exact_combine(s, c):
    out = torch.zeros(c["rows"], c["cols"], dtype=torch.float64, device="cuda")
    for i in range(c["k"]):
        out += s["gates"][:, i:i + 1].double() * s["y"][s["positions"][:, i].long()].double()
    return out if s["residual"] is None else out + s["residual"].double()
