"""The operators in 64 bits on the CPU, from their formulas, with bounds on
what fp32 sums and one rounding may add; and inputs for them."""

import math

import torch

U32 = 2.0 ** -24  # unit roundoffs
U16 = 2.0 ** -8   # bf16
U8 = 2.0 ** -4    # E4M3
TINY8 = 2.0 ** -10  # half the smallest E4M3 number

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f8e4m3": torch.float8_e4m3fn}
ROUND = {"f32": U32, "bf16": U16}


def blocks(cols):
    return -(-cols // 128)


def randn(*shape, seed=0, dtype="f32", scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g, dtype=torch.float64) * scale).to(TORCH[dtype])


def strided(t, pad, skip):
    """The same values on the GPU, rows ``pad`` elements further apart and
    ``skip`` elements into the buffer (off the 16-byte grid)."""
    rows, cols = t.shape
    buf = torch.empty(skip + rows * (cols + pad) + 8, dtype=t.dtype, device="cuda")
    view = buf[skip:skip + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    view.copy_(t.cuda())
    return view


def quant_rows(x):
    """(codes, scales) of rows, by torch's casts, as inputs."""
    rows, cols = x.shape
    p = torch.zeros(rows, blocks(cols) * 128)
    p[:, :cols] = x.float()
    p = p.view(rows, blocks(cols), 128)
    s = p.abs().amax(-1) / 448
    s = torch.where(s > 0, s, torch.ones_like(s))
    return (p / s[..., None]).view(rows, blocks(cols) * 128)[:, :cols].to(torch.float8_e4m3fn), s


def quant_blocks(w):
    n, k = w.shape
    p = torch.zeros(blocks(n) * 128, blocks(k) * 128)
    p[:n, :k] = w.float()
    p = p.view(blocks(n), 128, blocks(k), 128)
    s = p.abs().amax((1, 3)) / 448
    s = torch.where(s > 0, s, torch.ones_like(s))
    return (p / s[:, None, :, None]).view(blocks(n) * 128, -1)[:n, :k].to(torch.float8_e4m3fn), s


def spread(s, rows, cols, per_row):
    """Scales as wide as what they scale."""
    s = s.double().repeat_interleave(128, 1)[:, :cols]
    return s if per_row else s.repeat_interleave(128, 0)[:rows]


def check(got, want, err, what):
    """got within err (plus its type's rounding) of want; exact where want is
    not finite."""
    g = got.double().cpu()
    bound = err + ROUND["bf16" if got.dtype == torch.bfloat16 else "f32"] * (want.abs() + err) + 1e-38
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(g), torch.isnan(want)), f"{what}: NaN in other places"
    assert torch.equal(g[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)]), f"{what}: infinities"
    off = ((g - want).abs() - bound)[fine]
    assert off.numel() == 0 or off.max() <= 0, f"{what}: {float(off.max()):.3g} past the bound"


def check_f8(codes, scales, want, err, what):
    """codes [T, C] and scales against want: each scale is the largest
    magnitude of its columns over 448 within err, each code within half a
    step of want / scale."""
    rows, cols = want.shape
    c, s = codes.double().cpu(), scales.double().cpu()
    for b in range(blocks(cols)):
        w, e = want[:, b * 128:(b + 1) * 128], err[:, b * 128:(b + 1) * 128]
        top, room = w.abs().amax(1), e.amax(1)
        sc = s[:, b]
        zero = top == 0
        assert torch.all((sc - top / 448).abs()[~zero] <= ((room + top * 4 * U32) / 448)[~zero]), f"{what}: scale {b}"
        assert torch.all(sc[zero & (room == 0)] == 1.0), f"{what}: scale of zeros {b}"
        y = w / sc[:, None]
        bound = U8 * y.abs() + TINY8 + (e / sc[:, None]) * (1 + U8) + 4 * U32 * y.abs()
        off = (c[:, b * 128:(b + 1) * 128] - y).abs() - bound
        assert off.max() <= 0, f"{what}: codes of block {b}, {float(off.max()):.3g} past the bound"


def norm(x, weight, residual, eps):
    """(y, bound of y, total, bound of total)."""
    t = x.double() + (residual.double() if residual is not None else 0)
    cols = x.shape[1]
    inv = 1 / (t.pow(2).mean(1, keepdim=True) + eps).sqrt()
    y = t * inv * weight.double()
    # t is rounded once; the sum of squares over cols terms, the root and two products
    err = y.abs() * U32 * (cols + 16) + U32 * 4 * inv * weight.double().abs() * (
        x.double().abs() + (residual.double().abs() if residual is not None else 0))
    return y, err, t, t.abs() * U32


def act(z, kind):
    if kind == "silu":
        return z * torch.sigmoid(z)
    if kind == "gelu":
        return 0.5 * z * torch.erfc(-z / math.sqrt(2.0))
    return z


def product(x, w, bias, kind, gated, residual, xs=None, ws=None):
    """(out, bound) of rows x and one weight, any of them scaled codes."""
    xd, wd = x.double(), w.double()
    k = x.shape[1]
    if xs is not None:
        xd = xd * spread(xs, *x.shape, True)
        wd = wd * spread(ws, *w.shape, False)
    z = xd @ wd.T
    # a sum of k products in fp32, scaled, and a bias: every step is within one rounding of the magnitudes summed
    e = (xd.abs() @ wd.abs().T) * U32 * (k + 8)
    if bias is not None:
        z = z + bias.double()
        e = e + z.abs() * U32
    n = z.shape[1] // 2
    steep = 1.13  # the largest slope of silu and gelu
    if gated:
        g, u, eg, eu = z[:, :n], z[:, n:], e[:, :n], e[:, n:]
        a = act(g, kind)
        ea = steep * eg + a.abs() * 16 * U32 + g.abs() * 4 * U32
        out, e = a * u, ea * (u.abs() + eu) + a.abs() * eu + (a * u).abs() * U32
    else:
        out = act(z, kind)
        if kind != "none":
            e = steep * e + out.abs() * 16 * U32 + z.abs() * 4 * U32
    if residual is not None:
        out = out + residual.double()
        e = e + out.abs() * U32
    return out, e


def route(z, k, mask, renormalize):
    """Routing of logits by a loop over rows, in Python numbers."""
    rows, e = z.shape
    zd = z.double()
    experts = torch.full((rows, k), -1, dtype=torch.int64)
    gates = torch.zeros(rows, k, dtype=torch.float64)
    p_all = torch.zeros(rows, e, dtype=torch.float64)
    n = 0
    for t in range(rows):
        row = zd[t]
        if (mask is not None and not mask[t]) or not bool((row > -math.inf).any()):
            continue
        n += 1
        p = torch.softmax(row, 0)
        p_all[t] = p
        order = sorted((i for i in range(e) if row[i] > -math.inf), key=lambda i: (-float(row[i]), i))[:k]
        chosen = torch.softmax(row[order], 0) if renormalize else p[order]
        for i, x in enumerate(order):
            experts[t, i], gates[t, i] = x, chosen[i]
    places = sorted(((int(experts[t, i]), t, i) for t in range(rows) for i in range(k) if experts[t, i] >= 0))
    positions = torch.full((rows, k), -1, dtype=torch.int64)
    tokens = torch.full((rows * k,), -1, dtype=torch.int64)
    counts = torch.zeros(e, dtype=torch.int64)
    for at, (x, t, i) in enumerate(places):
        positions[t, i], tokens[at] = at, t
        counts[x] += 1
    offsets = torch.cat([torch.zeros(1, dtype=torch.int64), counts.cumsum(0)])
    loss = (counts.double() * p_all.sum(0)).sum() * e / (k * n * n) if n else torch.zeros((), dtype=torch.float64)
    return dict(experts=experts, gates=gates, positions=positions, tokens=tokens, counts=counts, offsets=offsets,
                loss=loss, routed=n, p=p_all)


def route_objective(z, r, k, renormalize, d_gates, d_loss):
    """What the gradient is of, with the choices fixed: a scalar in 64 bits of
    z [T, E] (rows that are sent nowhere, and -inf, give nothing)."""
    on = (r["experts"] >= 0).any(1)
    e = z.shape[1]
    p = torch.softmax(z, 1) * on[:, None]
    chosen = r["experts"].clamp(min=0)
    there = (r["experts"] >= 0).double()
    g = p.gather(1, chosen) * there
    if renormalize:
        g = g / torch.where(on[:, None], g.sum(1, keepdim=True), torch.ones_like(g[:, :1]))
    n = max(1, r["routed"])
    loss = (r["counts"].double() * p.sum(0)).sum() * e / (k * n * n)
    return (g * d_gates.double()).sum() + loss * d_loss
