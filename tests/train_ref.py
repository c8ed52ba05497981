"""The trainer's operators in 64 bits on the CPU, from their formulas, with
bounds on what fp32 may add: a product, a sum or a function off by its roundings,
a sum of n terms by its deepest chain of additions."""

import math

import torch

from ops_ref import U32, blocks


def depth(cols):
    """Additions that a term of a row's sum goes through at most: a lane's own, then lanes, wavefronts and steps."""
    return 128 + cols // 256


def embedding(tokens, weight, scale, first):
    """(out, bound)"""
    at = tokens.reshape(-1) - first
    there = (at >= 0) & (at < weight.shape[0])
    out = torch.zeros(len(at), weight.shape[1]).double()
    out[there] = weight.double()[at[there]] * scale
    out = out.view(*tokens.shape, weight.shape[1])
    return out, out.abs() * U32


def embedding_backward(d_out, tokens, rows, scale, first):
    at = tokens.reshape(-1) - first
    there = (at >= 0) & (at < rows)
    d = d_out.reshape(len(at), d_out.shape[-1]).double()
    total, size = torch.zeros(rows, d.shape[1]).double(), torch.zeros(rows, d.shape[1]).double()
    total.index_add_(0, at[there], d[there])
    size.index_add_(0, at[there], d[there].abs())
    n = torch.bincount(at[there], minlength=rows)[:, None]
    return total * scale, (size * (n + 1) + total.abs()) * U32 * abs(scale)


def layer_norm(x, weight, bias, residual, eps, center):
    """A dict of what the norm and its gradient are made of, with bounds e_*."""
    total = x if residual is None else (x.double() + residual.double()).float().to(residual.dtype)
    t, n = total.double(), x.shape[1]
    u = U32 * depth(n)
    mean = t.mean(1, keepdim=True) if center else torch.zeros(t.shape[0], 1).double()
    e_mean = (u + 2 * U32) * t.abs().mean(1, keepdim=True) if center else 0.0
    d = t - mean
    e_d = e_mean + U32 * d.abs()
    var = d.pow(2).mean(1, keepdim=True)
    e_var = (2 * d.abs() * e_d + e_d ** 2 if center else 0 * d).mean(1, keepdim=True) + (u + 4 * U32) * var
    inv = (var + eps).rsqrt()
    e_inv = inv * (0.5 * e_var / (var + eps) * (1 + 4 * e_var / (var + eps)) + 4 * U32)
    h = d * inv
    e_h = e_d * inv + d.abs() * e_inv + e_d * e_inv + U32 * h.abs()
    w = weight.double()
    out = h * w + (0 if bias is None else bias.double())
    return dict(total=total, mean=mean, inv=inv, h=h, out=out, e_h=e_h, e_inv=e_inv, e_mean=e_mean,
                e_out=e_h * w.abs() + U32 * out.abs())


def layer_norm_backward(f, weight, d_out, d_total, center):
    """(d_sum, bound), (d_weight, bound), (d_bias, bound) from layer_norm's dict."""
    d, w, h, e_h, inv, e_inv = d_out.double(), weight.double(), f["h"], f["e_h"], f["inv"], f["e_inv"]
    rows, n = d.shape
    u = U32 * depth(n)
    g = d * w
    e_g = g.abs() * U32
    c1 = g.mean(1, keepdim=True) if center else torch.zeros_like(inv)
    e_c1 = g.abs().mean(1, keepdim=True) * (u + 3 * U32) if center else torch.zeros_like(inv)
    c2 = (g * h).mean(1, keepdim=True)
    e_c2 = (g.abs() * e_h + e_g * (h.abs() + e_h)).mean(1, keepdim=True) + (g * h).abs().mean(1, keepdim=True) * (u + 3 * U32)
    s = g - c1 - h * c2
    e_s = e_g + e_c1 + h.abs() * e_c2 + e_h * (c2.abs() + e_c2) + 3 * U32 * (g.abs() + c1.abs() + (h * c2).abs())
    ds = inv * s
    e = e_inv * (s.abs() + e_s) + inv * e_s + U32 * ds.abs()
    if d_total is not None:
        ds = ds + d_total.double()
        e = e + U32 * ds.abs()
    ends = rows + 16
    dw, e_dw = (d * h).sum(0), (d.abs() * e_h).sum(0) + (d * h).abs().sum(0) * U32 * ends
    db, e_db = d.sum(0), d.abs().sum(0) * U32 * ends
    return (ds, e), (dw, e_dw), (db, e_db)


def own(routing, span):
    """Whether each choice's place is one that counts."""
    p = routing["positions"]
    lo, hi = (0, len(routing["tokens"])) if span is None else (max(0, span[0]), min(span[1], len(routing["tokens"])))
    return (p >= lo) & (p < hi)


def dispatch(x, routing, span):
    out = torch.zeros(len(routing["tokens"]), x.shape[1], dtype=x.dtype)
    there = own(routing, span)
    row = torch.arange(x.shape[0])[:, None].expand(there.shape)
    out[routing["positions"][there]] = x[row[there]]
    return out


def dispatch_backward(d, routing, span):
    there = own(routing, span)
    rows = d.double()[routing["positions"].clamp(min=0)] * there[..., None]
    return rows.sum(1), rows.abs().sum(1) * U32 * there.shape[1]


def collect_backward(d_out, y, routing, gates, span):
    """(d_y, bound), (d_gates, bound)"""
    there = own(routing, span)
    row = torch.arange(there.shape[0])[:, None].expand(there.shape)[there]
    place, g = routing["positions"][there], gates.double()[there][:, None]
    d_y, d_g, e_g = torch.zeros(y.shape).double(), torch.zeros(there.shape).double(), torch.zeros(there.shape).double()
    d_y[place] = g * d_out.double()[row]
    terms = d_out.double()[row] * y.double()[place]
    d_g[there], e_g[there] = terms.sum(1), terms.abs().sum(1) * U32 * depth(y.shape[1])
    return (d_y, d_y.abs() * U32), (d_g, e_g)


def curve(z, kind):
    """(act(z), bound, slope, bound) of an exact z."""
    if kind == "none":
        return z, 0 * z, torch.ones_like(z), 0 * z
    if kind == "silu":
        p, q = torch.sigmoid(z), torch.sigmoid(-z)
        a = z * p
        return a, a.abs() * 16 * U32, p + a * q, (p + (a * q).abs()) * 16 * U32
    # erfc's and e^'s argument is rounded, which z^2 of its roundings go over into the result
    below, hill = 0.5 * torch.erfc(-z / math.sqrt(2.0)), z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    a, steps = z * below, (16 + 2 * z * z) * U32
    return a, a.abs() * steps, below + hill, (below + hill.abs()) * steps


def kept(x, gated):
    """(codes, scales) of x in 8 bits."""
    codes, scales = [], []
    for half in x.float().chunk(2, 1) if gated else [x.float()]:
        for b in half.split(128, 1):
            s = b.abs().amax(1, keepdim=True)
            s = s / torch.full_like(s, 448)
            s = torch.where(s > 0, s, torch.ones_like(s))
            codes.append((b / s).to(torch.float8_e4m3fn).view(torch.uint8))
            scales.append(s)
    return torch.cat(codes, 1).view(torch.float8_e4m3fn), torch.cat(scales, 1)


def kept_values(codes, scales, gated):
    n = codes.shape[1] // 2 if gated else codes.shape[1]
    s = [p.double().repeat_interleave(128, 1)[:, :n] for p in scales.split(blocks(n), 1)]
    return codes.double() * torch.cat(s, 1)


def activate(x, kind, gated):
    """(out, bound)"""
    if not gated:
        return curve(x.double(), kind)[:2]
    g, up = x.double().chunk(2, 1)
    a, e, _, _ = curve(g, kind)
    return a * up, e * up.abs() + (a * up).abs() * U32


def activate_backward(d_out, z, kind, gated, off=0.0):
    """(d_x, bound) at the values z, themselves off by ``off`` of their size."""
    d = d_out.double()
    steep = 1.13  # the largest slope, and more than the largest change of a slope with z
    if not gated:
        _, _, s, e = curve(z, kind)
        return d * s, d.abs() * (e + off * z.abs() * steep) + (d * s).abs() * U32
    g, up = z.chunk(2, 1)
    a, e_a, s, e_s = curve(g, kind)
    e_a, e_s = e_a + off * g.abs() * steep, e_s + off * g.abs() * steep
    d_g, d_up = d * up * s, d * a
    return (torch.cat([d_g, d_up], 1),
            torch.cat([(d * up).abs() * (e_s * (1 + off) + s.abs() * off) + d_g.abs() * 3 * U32, d.abs() * e_a + d_up.abs() * U32], 1))
