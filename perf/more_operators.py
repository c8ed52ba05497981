"""Timed cases of the trainer's operators around an MoE layer's products: the
lookup of token embeddings and its gradient, layer norm of a residual sum, rows
sorted by expert and back, and the activation with a checkpoint in 8 bits.

A case names one operator (``op``) and its sizes; with ``step`` a pass is the
operator and its gradient, else the operator alone:

* ``embed``    ``rows`` tokens looked up in a table of ``vocab`` rows (with
               ``shard`` the upper half of a vocabulary of twice as many);
* ``norm``     ``rows`` tokens of ``cols`` values added to a residual (of type
               ``stream``, or none) and normed, centred or not;
* ``dispatch`` ``rows`` tokens copied to their ``k`` experts' places;
* ``collect``  ``rows`` tokens, each the weighted sum of its ``k`` expert rows;
* ``act``      ``rows`` tokens of ``cols`` activations, gated or not, with the
               input kept in 8 bits for the gradient (``keep``) or as it is.

8-bit checkpoints are E4M3 values with an fp32 scale per 128 values of a row
(of each of its halves, gate and up).
"""

import math
import random

import torch

own = False

EPS = 1e-5
BLOCK = 128
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"bf16": 2, "f32": 4}


def listed():
    return [
        # the next token of one sequence: the call is what costs
        dict(name="embed_token", op="embed", rows=1, vocab=32000, cols=4096, dtype="bf16", shard=False, scaled=False,
             step=False),
        # a training microbatch with the table's whole gradient
        dict(name="embed_train", op="embed", rows=16384, vocab=128256, cols=4096, dtype="bf16", shard=False,
             scaled=False, step=True),
        # a rank with half of a vocabulary, scaled lookups, fp32, no size a multiple of anything
        dict(name="embed_shard", op="embed", rows=3001, vocab=16013, cols=1499, dtype="f32", shard=True, scaled=True,
             step=True),
        # one decode step of one sequence
        dict(name="norm_token", op="norm", rows=1, cols=7168, dtype="bf16", stream="bf16", center=True, bias=True,
             step=False),
        # a training microbatch, the residual's gradient coming in beside the norm's
        dict(name="norm_train", op="norm", rows=16384, cols=4096, dtype="bf16", stream="bf16", center=True, bias=True,
             step=True),
        # an uncentred norm on an fp32 residual stream, odd sizes
        dict(name="norm_ragged", op="norm", rows=1777, cols=1501, dtype="bf16", stream="f32", center=False, bias=False,
             step=True),
        # a decode step of 32 sequences, eight experts
        dict(name="dispatch_decode", op="dispatch", rows=32, cols=4096, experts=8, k=2, dtype="bf16", mask=False,
             step=False),
        # a training microbatch with padding, 256 experts
        dict(name="dispatch_train", op="dispatch", rows=8192, cols=7168, experts=256, k=8, dtype="bf16", mask=True,
             step=True),
        # a small fp32 batch of odd sizes
        dict(name="collect_ragged", op="collect", rows=333, cols=1111, experts=12, k=3, dtype="f32", mask=True,
             residual=True, step=True),
        # the way back of the training microbatch
        dict(name="collect_train", op="collect", rows=8192, cols=7168, experts=256, k=8, dtype="bf16", mask=True,
             residual=True, step=True),
        # a dense layer's gelu on few tokens, its input kept as it is
        dict(name="act_few", op="act", rows=24, cols=4097, dtype="f32", kind="gelu", gated=False, keep=False, step=True),
        # gate and up of a training microbatch, kept in 8 bits
        dict(name="act_train", op="act", rows=8192, cols=14336, dtype="bf16", kind="silu", gated=True, keep=True,
             step=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A length of the range: as drawn in a third of the cases, else a multiple of 64."""
    n = _log(rng, lo, hi)
    return n if rng.random() < 0.35 else max(64, n // 64 * 64)


def draw(rng):
    """A case of the same kinds: one to tens of thousands of rows, narrow to wide, plain and odd sizes."""
    most = max(work(c)["bytes"] for c in listed())
    while True:
        op = rng.choice(["embed", "norm", "dispatch", "collect", "act"])
        c = dict(op=op, rows=_log(rng, 1, 16384), cols=_size(rng, 64, 14336 if op == "act" else 8192),
                 dtype=rng.choice(["bf16", "bf16", "f32"]), step=rng.random() < 0.75)
        if op == "embed":
            c.update(vocab=_log(rng, 100, 131072), shard=rng.random() < 0.3, scaled=rng.random() < 0.5)
        elif op == "norm":
            c.update(stream=rng.choice(["bf16", "bf16", "f32", None]), center=rng.random() < 0.6)
            c.update(bias=c["center"] and rng.random() < 0.7)
        elif op == "act":
            gated = rng.random() < 0.6
            c.update(gated=gated, kind=rng.choice(["silu", "gelu"]), keep=rng.random() < 0.6)
        else:
            experts = rng.choice([8, 16, 64, 256, _log(rng, 2, 512)])
            c.update(experts=experts, k=rng.randint(1, min(8, experts)), mask=rng.random() < 0.5)
            if op == "collect":
                c.update(residual=rng.random() < 0.6)
        if work(c)["bytes"] <= most:
            return c


def work(c):
    rows, cols, es, step = c["rows"], c["cols"], BYTES[c["dtype"]], c["step"]
    n = rows * cols
    if c["op"] == "embed":
        # tokens are 8 bytes; a lookup reads a table's row at most once
        there = 8 * rows + es * (min(rows, c["vocab"]) * cols + n)
        back = 8 * rows + es * (n + c["vocab"] * cols)
        return {"bytes": there + (back if step else 0), "flops": n * (2 if step else 1)}
    if c["op"] == "norm":
        s = BYTES[c["stream"]] if c["stream"] else 0
        ts = s or es  # the type of what is normed
        there = n * (2 * es + 2 * s) + (8 if c["center"] else 4) * rows + es * cols * (1 + c["bias"])
        dx = es if not s or s == es else es + s  # two results where the sum's parts have different types
        back = n * (ts + es + s + dx) + (8 if c["center"] else 4) * rows + es * cols * (2 + c["bias"])
        return {"bytes": there + (back if step else 0), "flops": n * (20 if step else 7)}
    if c["op"] == "dispatch":
        k = c["k"]
        there = es * n * (1 + k) + 4 * rows * k
        back = es * n * (k + 1) + 4 * rows * k
        return {"bytes": there + (back if step else 0), "flops": n * k if step else 0}
    if c["op"] == "collect":
        k = c["k"]
        there = es * n * (k + 1 + c["residual"]) + 8 * rows * k
        back = es * n * (1 + 2 * k) + 16 * rows * k
        return {"bytes": there + (back if step else 0), "flops": n * k * (5 if step else 2)}
    wide = n * (2 if c["gated"] else 1)
    blocks = rows * -(-cols // BLOCK) * (2 if c["gated"] else 1)
    held = wide + 4 * blocks if c["keep"] else wide * es
    there = es * (wide + n) + (held if c["keep"] else 0)
    back = held + es * (n + wide)
    return {"bytes": there + (back if step else 0), "flops": n * (30 if step else 10)}


# ---- inputs ------------------------------------------------------------------------------------


def _activations(g, rows, cols, dtype):
    """Hidden states: a few columns are much larger than the others, as in trained models."""
    x = torch.randn(rows, cols, generator=g, device="cuda")
    x.mul_(torch.rand(cols, generator=g, device="cuda").mul_(3).exp_().mul_(0.3))
    return x.to(TYPES[dtype])


def _gradients(g, rows, cols, dtype):
    return torch.randn(rows, cols, generator=g, device="cuda").to(TYPES[dtype])


def _tokens(g, rows, vocab):
    """Token ids as texts have them: the r-th most frequent about 1 / r as often as the first; a tenth is padding."""
    rank = torch.rand(rows, generator=g, device="cuda", dtype=torch.float64).mul_(math.log(vocab)).exp_().long() - 1
    ids = torch.randperm(vocab, generator=g, device="cuda")[rank.clamp_(0, vocab - 1)]
    return torch.where(torch.rand(rows, generator=g, device="cuda") < 0.1, 0, ids)


def _routing(g, c):
    """A routing as the router leaves it: experts differ in how often they are chosen, masked rows go nowhere."""
    rows, experts, k = c["rows"], c["experts"], c["k"]
    z = torch.randn(rows, experts, generator=g, device="cuda").add_(torch.randn(experts, generator=g, device="cuda").mul_(0.5))
    top, chosen = z.topk(k, -1)
    gates = torch.softmax(top, -1)
    on = torch.ones(rows, dtype=torch.bool, device="cuda")
    if c["mask"]:
        on = torch.rand(rows, generator=g, device="cuda") < 0.9
        chosen, gates = torch.where(on[:, None], chosen, experts), gates * on[:, None]
    flat = chosen.reshape(-1)
    place = torch.sort(flat, stable=True)[1]
    here = torch.arange(rows * k, device="cuda")
    positions = torch.empty_like(place)
    positions[place] = here
    positions = torch.where(flat == experts, -1, positions).view(rows, k)
    counts = torch.bincount(flat, minlength=experts + 1)[:experts]
    offsets = torch.cat([counts.new_zeros(1), counts.cumsum(0)])
    tokens = torch.where(here < offsets[-1], place // k, -1)
    return dict(experts=torch.where(chosen == experts, -1, chosen).int(), gates=gates, positions=positions.int(),
                tokens=tokens.int(), counts=counts.int(), offsets=offsets.int(), loss=torch.zeros((), device="cuda"),
                routed=on.sum().int().view(1), mask=None, renormalize=True)


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda").manual_seed(seed)
    rows, cols, t = c["rows"], c["cols"], c["dtype"]
    if c["op"] == "embed":
        s = dict(tokens=_tokens(g, rows, c["vocab"] * (2 if c["shard"] else 1)),
                 weight=torch.randn(c["vocab"], cols, generator=g, device="cuda", dtype=torch.bfloat16).mul_(0.02).to(TYPES[t]),
                 first=c["vocab"] if c["shard"] else 0, scale=math.sqrt(cols) if c["scaled"] else 1.0)
        if c["step"]:
            s["d_out"] = _gradients(g, rows, cols, t)
    elif c["op"] == "norm":
        s = dict(x=_activations(g, rows, cols, t), residual=None, bias=None,
                 weight=(1 + 0.1 * torch.randn(cols, generator=g, device="cuda")).to(TYPES[t]))
        if c["bias"]:
            s["bias"] = (0.1 * torch.randn(cols, generator=g, device="cuda")).to(TYPES[t])
        if c["stream"]:
            s["residual"] = _activations(g, rows, cols, c["stream"])
        if c["step"]:
            s.update(d_out=_gradients(g, rows, cols, t),
                     d_total=_gradients(g, rows, cols, c["stream"]) if c["stream"] else None)
    elif c["op"] == "act":
        s = dict(x=_activations(g, rows, cols * (2 if c["gated"] else 1), t))
        if c["step"]:
            s["d_out"] = _gradients(g, rows, cols, t)
    else:
        s = dict(routing=_routing(g, c))
        if c["op"] == "dispatch":
            s["x"] = _activations(g, rows, cols, t)
            if c["step"]:
                s["d_rows"] = _gradients(g, rows * c["k"], cols, t)
        else:
            s.update(y=_activations(g, rows * c["k"], cols, t),
                     residual=_activations(g, rows, cols, t) if c["residual"] else None)
            if c["step"]:
                s["d_out"] = _gradients(g, rows, cols, t)
    s["case"] = c
    return s


def run(state):
    return (_run_own if own else _run_plain)(state)


# ---- the framework's calls ---------------------------------------------------------------------


def _run_own(s):
    import paper_2609_25442_amd as wb

    c = s["case"]
    step = c["step"]
    if c["op"] == "embed":
        got = [wb.embedding(s["tokens"], s["weight"], scale=s["scale"], first=s["first"])]
        if step:
            got.append(wb.embedding_backward(s["d_out"], s["tokens"], c["vocab"], scale=s["scale"], first=s["first"]))
        return got
    if c["op"] == "norm":
        n = wb.add_layer_norm(s["x"], s["weight"], s["bias"], s["residual"], eps=EPS, center=c["center"])
        got = [n.out] if s["residual"] is None else [n.out, n.total]
        if step:
            d = wb.add_layer_norm_backward(s["d_out"], n, s["weight"], d_total=s["d_total"])
            got += [v for v in (d.x, d.residual, d.weight, d.bias) if v is not None]
        return got
    if c["op"] == "act":
        a = wb.activate(s["x"], c["kind"], gated=c["gated"], checkpoint=c["keep"])
        return [a.out, wb.activate_backward(s["d_out"], a)] if step else [a.out]
    r = wb.Routing(**s["routing"])
    if c["op"] == "dispatch":
        got = [wb.dispatch(s["x"], r)]
        if step:
            got.append(wb.dispatch_backward(s["d_rows"], r))
        return got
    got = [wb.collect(s["y"], r, residual=s["residual"])]
    if step:
        got += wb.collect_backward(s["d_out"], s["y"], r)
    return got


# ---- the plain forms: elementary operations in 32 bits -----------------------------------------


def _run_plain(s):
    return {"embed": _plain_embed, "norm": _plain_norm, "dispatch": _plain_dispatch, "collect": _plain_collect,
            "act": _plain_act}[s["case"]["op"]](s, s["case"])


def _plain_embed(s, c):
    w = s["weight"]
    at = s["tokens"] - s["first"]
    there = (at >= 0) & (at < c["vocab"])
    at = torch.where(there, at, 0)
    got = [(w[at].float() * s["scale"] * there[:, None]).to(w.dtype)]
    if c["step"]:
        d = torch.zeros(w.shape, device=w.device)
        d.index_add_(0, at, s["d_out"].float() * there[:, None])
        got.append((d * s["scale"]).to(w.dtype))
    return got


def _plain_norm(s, c):
    x, r, w = s["x"], s["residual"], s["weight"].float()
    total = x if r is None else (x.float() + r.float()).to(r.dtype)
    t = total.float()
    if c["center"]:
        t = t - t.mean(-1, keepdim=True)
    inv = torch.rsqrt((t * t).mean(-1, keepdim=True) + EPS)
    t = t * inv
    y = t * w
    if s["bias"] is not None:
        y = y + s["bias"].float()
    got = [y.to(x.dtype)] if r is None else [y.to(x.dtype), total]
    if c["step"]:
        d = s["d_out"].float()
        dw = (d * t).sum(0)
        g = d * w
        dt = g - t * (g * t).mean(-1, keepdim=True)
        if c["center"]:
            dt = dt - g.mean(-1, keepdim=True)
        dt = dt * inv
        if r is not None:
            dt = dt + s["d_total"].float()
        got.append(dt.to(x.dtype))
        if r is not None:
            got.append(dt.to(r.dtype))
        got.append(dw.to(x.dtype))
        if s["bias"] is not None:
            got.append(d.sum(0).to(x.dtype))
    return got


def _plain_dispatch(s, c):
    x, tokens, positions = s["x"], s["routing"]["tokens"].long(), s["routing"]["positions"].long()
    got = [torch.where(tokens[:, None] >= 0, x[tokens.clamp(min=0)], 0)]
    if c["step"]:
        rows = s["d_rows"][positions.clamp(min=0)].float() * (positions >= 0)[..., None]
        got.append(rows.sum(1).to(x.dtype))
    return got


def _plain_collect(s, c):
    y, tokens, positions = s["y"], s["routing"]["tokens"].long(), s["routing"]["positions"].long()
    gates = s["routing"]["gates"]
    there = positions >= 0
    at = positions.clamp(min=0)
    rows = y[at].float() * there[..., None]
    out = (rows * gates[..., None]).sum(1)
    if s["residual"] is not None:
        out = out + s["residual"].float()
    got = [out.to(y.dtype)]
    if c["step"]:
        d = s["d_out"].float()
        by_place = torch.zeros(y.shape[0] + 1, device=y.device)
        by_place[torch.where(there, positions, y.shape[0])] = gates
        dy = d[tokens.clamp(min=0)] * (by_place[:-1] * (tokens >= 0))[:, None]
        got += [dy.to(y.dtype), (rows * d[:, None]).sum(-1)]
    return got


def _in_8_bits(x):
    """The values that stand for the fp32 rows x in E4M3 with a scale per 128 columns."""
    rows, cols = x.shape
    nb = -(-cols // BLOCK)
    p = torch.zeros(rows, nb * BLOCK, device=x.device)
    p[:, :cols] = x
    p = p.view(rows, nb, BLOCK)
    s = p.abs().amax(-1, keepdim=True)
    s = s / torch.full_like(s, 448)  # a quotient: values lie on borders of E4M3 that a product with 1 / 448 would move
    s = torch.where(s > 0, s, torch.ones_like(s))
    return ((p / s).to(torch.float8_e4m3fn).float() * s).view(rows, -1)[:, :cols]


def _act_and_slope(z, kind):
    if kind == "silu":
        s = 1 / (1 + torch.exp(-z))
        return z * s, s * (1 + z * (1 - s))
    below = 0.5 * torch.erfc(z * -math.sqrt(0.5))
    return z * below, below + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))


def _plain_act(s, c):
    x = s["x"]
    parts = [p.float() for p in (x.chunk(2, -1) if c["gated"] else (x,))]
    a, _ = _act_and_slope(parts[0], c["kind"])
    got = [(a * parts[1] if c["gated"] else a).to(x.dtype)]
    if c["step"]:
        d = s["d_out"].float()
        if c["keep"]:
            parts = [_in_8_bits(p) for p in parts]
        a, slope = _act_and_slope(parts[0], c["kind"])
        d = torch.cat([d * parts[1] * slope, d * a], -1) if c["gated"] else d * slope
        got.append(d.to(x.dtype))
    return got


# ---- the definitions in 64 bits ----------------------------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    return {"embed": _exact_embed, "norm": _exact_norm, "dispatch": _exact_dispatch, "collect": _exact_collect,
            "act": _exact_act}[case["op"]](s, case)


def _exact_embed(s, c):
    table = torch.cat([s["weight"].double(), torch.zeros(1, c["cols"], dtype=torch.float64, device="cuda")])
    at = s["tokens"] - s["first"]
    at[(at < 0) | (at >= c["vocab"])] = c["vocab"]  # the row of zeros
    got = [table[at] * s["scale"]]
    if c["step"]:
        table.zero_()
        table.index_put_((at,), s["d_out"].double() * s["scale"], accumulate=True)
        got.append(table[:-1])
    return got


def _exact_norm(s, c):
    x, r = s["x"].double(), s["residual"]
    total = x if r is None else x + r.double()
    t = total if r is None else total.to(r.dtype).double()  # the norm is of the sum as it is kept
    n = c["cols"]
    mu = t.sum(1, keepdim=True) / n if c["center"] else torch.zeros_like(t[:, :1])
    sigma = (((t - mu) ** 2).sum(1, keepdim=True) / n + EPS).sqrt()
    hat, w = (t - mu) / sigma, s["weight"].double()
    got = [hat * w + (0 if s["bias"] is None else s["bias"].double())] + ([] if r is None else [total])
    if c["step"]:
        d = s["d_out"].double()
        of_hat = d * w
        along = (of_hat * hat).sum(1, keepdim=True) / n
        down = of_hat.sum(1, keepdim=True) / n if c["center"] else 0
        dt = (of_hat - down - hat * along) / sigma
        if r is not None:
            dt = dt + s["d_total"].double()
        got += [dt] if r is None else [dt, dt]
        got.append((d * hat).sum(0))
        if s["bias"] is not None:
            got.append(d.sum(0))
    return got


def _choices(s, c):
    """(row, place) of every choice, by rows."""
    positions = s["routing"]["positions"].long()
    row, i = torch.nonzero(positions >= 0, as_tuple=True)
    return row, i, positions[row, i]


def _exact_dispatch(s, c):
    row, _, place = _choices(s, c)
    x = s["x"].double()
    rows = torch.zeros(c["rows"] * c["k"], c["cols"], dtype=torch.float64, device="cuda")
    rows[place] = x[row]
    got = [rows]
    if c["step"]:
        d = torch.zeros_like(x)
        d.index_add_(0, row, s["d_rows"][place].double())
        got.append(d)
    return got


def _exact_collect(s, c):
    row, i, place = _choices(s, c)
    gate = s["routing"]["gates"].double()[row, i][:, None]
    out = torch.zeros(c["rows"], c["cols"], dtype=torch.float64, device="cuda")
    out.index_add_(0, row, gate * s["y"][place].double())
    if s["residual"] is not None:
        out += s["residual"].double()
    got = [out]
    if c["step"]:
        d = s["d_out"].double()[row]
        dy = torch.zeros(c["rows"] * c["k"], c["cols"], dtype=torch.float64, device="cuda")
        dy[place] = gate * d
        dg = torch.zeros(c["rows"], c["k"], dtype=torch.float64, device="cuda")
        dg[row, i] = (d * s["y"][place].double()).sum(1)
        got += [dy, dg]
    return got


def _exact_kept(x):
    """What a half's rows are kept as: a scale is an fp32 number, and so is what is rounded to E4M3."""
    kept = []
    for b in x.split(BLOCK, 1):
        top = (b.abs().amax(1, keepdim=True).double() / 448).float().double()
        top[top == 0] = 1
        kept.append((b.double() / top).float().to(torch.float8_e4m3fn).double() * top)
    return torch.cat(kept, 1)


def _exact_slope(z, kind):
    if kind == "silu":
        return torch.sigmoid(z) * (1 + z * torch.sigmoid(-z))
    return 0.5 * torch.erfc(-z / math.sqrt(2.0)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)


def _exact_value(z, kind):
    return z * torch.sigmoid(z) if kind == "silu" else z * 0.5 * torch.erfc(-z / math.sqrt(2.0))


def _exact_act(s, c):
    parts = s["x"].chunk(2, 1) if c["gated"] else [s["x"]]
    z = _exact_value(parts[0].double(), c["kind"])
    got = [z * parts[1].double() if c["gated"] else z]
    if c["step"]:
        d = s["d_out"].double()
        gate, *up = [_exact_kept(p) if c["keep"] else p.double() for p in parts]
        if up:
            got.append(torch.cat([d * up[0] * _exact_slope(gate, c["kind"]), d * _exact_value(gate, c["kind"])], 1))
        else:
            got.append(d * _exact_slope(gate, c["kind"]))
    return got
