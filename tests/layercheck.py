"""The operators around attention (embeddings, norms of rows, gated MLP, log probabilities) in 64 bits on the CPU, from their formulas, and how far an
implementation that rounds where the header says may be from them.  `u` of opscheck is half a step of a type."""
import math

import torch

from opscheck import F64, U32, assert_near, d, rounding, u  # noqa: F401

TINY = torch.finfo(torch.float32).tiny


def f32(x):
    """A number as the library takes it."""
    return float(torch.tensor(x, dtype=torch.float32))


# ----------------------------------------------------------------------------------------------------------- embeddings
def embed(ids, table, scale):
    """(out, tolerance): one product in 32 bits, one rounding"""
    ids, t = ids.cpu().long(), d(table)
    fine = (ids >= 0) & (ids < t.shape[0])
    y = t[ids.clamp(0, t.shape[0] - 1)] * f32(scale)
    y = torch.where(fine[..., None], y, math.nan)
    y0 = torch.nan_to_num(y)
    return y, rounding(y0, table.dtype) + U32 * y0.abs()


def embed_backward(dout, ids, rows, scale):
    """A row's terms are added in 32 bits, each addition off by U32 of a sum no larger than the magnitudes' sum; then the product and a rounding."""
    ids, g = ids.cpu().long().flatten(), d(dout).reshape(-1, dout.shape[-1])
    fine = (ids >= 0) & (ids < rows)
    ids, g = ids[fine], g[fine]
    sums, mags = (torch.zeros(rows, g.shape[1], dtype=F64).index_add_(0, ids, x) for x in (g, g.abs()))
    n = torch.bincount(ids, minlength=rows)[:, None]
    y = sums * f32(scale)
    return y, rounding(y, dout.dtype) + (n + 1) * U32 * mags * abs(f32(scale))


# -------------------------------------------------------------------------------------------------------- norms of rows
def norm(x, weight, bias, eps, center, dtype, dy=None):
    """{name: (value, tolerance)}: y, or dx, dweight and dbias."""
    dim = x.shape[-1]
    x, dy = d(x).reshape(-1, dim), None if dy is None else d(dy).reshape(-1, dim)            # (values come as rows)
    w = torch.ones(dim, dtype=F64) if weight is None else d(weight)
    b = torch.zeros(dim, dtype=F64) if bias is None else d(bias)
    m = x.mean(-1, keepdim=True) if center else torch.zeros_like(x[..., :1])
    c = x - m
    r = 1 / (c.square().mean(-1, keepdim=True) + f32(eps)).sqrt()
    n = c * r
    # the mean: dim additions; what is left of a value is off by the mean's error and its own rounding; the sum of squares (dim additions, half
    # of which reach the root), root, division and the products
    em = (dim + 1) * U32 * x.abs().mean(-1, keepdim=True) if center else 0.0 * r
    rel = em * r + (dim / 2 + 8) * U32
    en = em * r + n.abs() * rel
    if dy is None:
        y = n * w + b
        return {"y": (y, rounding(y, dtype) + w.abs() * en + 2 * U32 * ((n * w).abs() + b.abs()))}
    g, gw = dy, dy * w
    dot, off = (gw * n).mean(-1, keepdim=True), gw.mean(-1, keepdim=True) if center else 0.0 * r
    dx = r * (gw - n * dot - off)
    edot = (gw.abs() * en).mean(-1, keepdim=True) + (dim + 4) * U32 * (gw * n).abs().mean(-1, keepdim=True)
    eoff = (dim + 4) * U32 * gw.abs().mean(-1, keepdim=True) if center else 0.0 * r
    mag = r * (gw.abs() + (n * dot).abs() + off.abs())
    rows = x.shape[0]
    dw, db = (g * n).sum(0), g.sum(0)
    out = {"dx": (dx, rounding(dx, dtype) + (rel + 6 * U32) * mag + r * (n.abs() * edot + en * dot.abs() + eoff))}
    if weight is not None:
        out["dweight"] = dw, rounding(dw, weight.dtype) + (g.abs() * en).sum(0) + (rows + 4) * U32 * (g * n).abs().sum(0)
    if bias is not None:
        out["dbias"] = db, rounding(db, bias.dtype) + (rows + 4) * U32 * g.abs().sum(0)
    return out


# ----------------------------------------------------------------------------------------------------------- gated MLP
def gated(x, gate, up, act, dh=None):
    """{name: (value, tolerance)}: h, or dx, dgate and dup."""
    dtype, e = x.dtype, u(x.dtype)
    x, wg, wu = d(x).reshape(-1, x.shape[-1]), d(gate), d(up)
    k = x.shape[1]
    g, v = x @ wg, x @ wu
    eg, ev = (k + 2) * U32 * (x.abs() @ wg.abs()), (k + 2) * U32 * (x.abs() @ wu.abs())     # sums of k products in any order
    # the share of g that passes, its slope; both are off by their arguments' errors (slopes up to 1.13 and 0.8) and by the exponential's or error
    # function's, whose argument is rounded first
    if act == "silu":
        s = torch.sigmoid(g)
        slope, ef = s * (1 + g * (1 - s)), (2 * g.abs() + 8) * U32
    else:
        s = torch.special.ndtr(g)
        slope, ef = s + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi), (g * g + 16) * U32
    a = g * s
    ea, es = 1.13 * eg + ef * a.abs() + TINY, 0.8 * eg + 2 * ef * (s + (slope - s).abs() + g.abs() * s * (1 - s)) + TINY
    if dh is None:
        h = a * v
        return {"h": (h, rounding(h, dtype) + v.abs() * ea + a.abs() * ev + ea * ev + 2 * U32 * h.abs())}
    dh = d(dh).reshape(-1, dh.shape[-1])
    dg, du = dh * v * slope, dh * a
    tg = rounding(dg, dtype) + (1 + e) * (dh.abs() * (ev * slope.abs() + v.abs() * es + ev * es) + 3 * U32 * dg.abs())
    tu = rounding(du, dtype) + (1 + e) * (dh.abs() * ea + 2 * U32 * du.abs())
    dx = dg @ wg.T + du @ wu.T
    n, rows = wg.shape[1], x.shape[0]
    out = {"dx": (dx, rounding(dx, dtype) + tg @ wg.abs().T + tu @ wu.abs().T + (2 * n + 2) * U32 * ((dg.abs() + tg) @ wg.abs().T + (du.abs() + tu) @ wu.abs().T))}
    for name, z, t in (("dgate", dg, tg), ("dup", du, tu)):
        y = x.T @ z
        out[name] = y, rounding(y, dtype) + x.abs().T @ t + (rows + 2) * U32 * (x.abs().T @ (z.abs() + t))
    return out


def assert_gated(got, want, dtype):
    """Each value within its bound; and all together: the errors are those of two roundings (of dg and du, and of the result), each at most u of
    its value and none depending on another, which do not grow in the norm over a sum: 2 u of the result's norm."""
    for n, (y, t) in want.items():
        x = d(got[n]).reshape(y.shape)
        assert_near(x, y, t, n)
        if y.numel():
            off, size = float((x - y).norm()), float(y.norm())
            assert off <= 2 * u(dtype) * size + float(rounding(torch.zeros_like(y), dtype).norm()) + 1e-30, (n, off, size)


# ---------------------------------------------------------------------------------------------------- log probabilities
def log_probs(logits, tokens, scale, ignore, top=0, dlogp=None, dentropy=None):
    """{name: (value, tolerance)}, and the ids of the top by value and place."""
    dtype, v, sc = logits.dtype, logits.shape[-1], f32(scale)
    x = d(logits).reshape(-1, v)
    z = x * sc
    m = z.amax(-1, keepdim=True)
    none = m == -math.inf
    dd = torch.where(z == -math.inf, 0.0, z - torch.where(none, 0.0, m))                      # distances of what has a probability
    e = torch.where(z == -math.inf, 0.0, torch.exp(dd))
    s = e.sum(-1, keepdim=True)
    ls = torch.log(torch.where(none, 1.0, s))
    lse = torch.where(none, -math.inf, m + ls)
    p = e / torch.where(none, 1.0, s)
    lp = torch.where(z == -math.inf, -math.inf, z - torch.where(none, 0.0, lse))
    # an exponential: its argument's difference, product and rounding (4 of it), itself 4; the sum: v additions; a sum is scaled when the maximum
    # moves, off by the distance moved, all of them together by no more than the range of what has a share
    rang = torch.where(e > 0, dd.abs(), 0.0).amax(-1, keepdim=True)
    es = (v + 64 + 8 * rang) * U32
    fin = lambda t: torch.where(torch.isfinite(t), t, 0.0).abs()                              # noqa: E731
    tl = es + 4 * U32 * (fin(m) + fin(lse) + 1)
    out = {"lse": (lse[:, 0], tl[:, 0])}
    far = (p * dd.abs()).sum(-1, keepdim=True)
    ent = torch.where(none, 0.0, ls + far)
    te = 2 * es * (1 + far + ls.abs())
    out["entropy"] = ent[:, 0], te[:, 0]
    t = hit = None
    if tokens is not None:
        t = tokens.reshape(-1).cpu().long()
        skip, inside = t == ignore, (t >= 0) & (t < v)
        hit = (inside & ~skip)[:, None]
        at = t.clamp(0, v - 1)[:, None]
        logp = torch.where(skip[:, None], 0.0, torch.where(hit, lp.gather(1, at), math.nan))
        tz = tl + 4 * U32 * (fin(z.gather(1, at)) + fin(lse))
        out["logp"] = logp[:, 0], torch.where(hit, tz, 0.0)[:, 0]
    ids = None
    if top:
        ids = torch.sort(x, dim=-1, descending=True, stable=True)[1][:, :top]
        out["top_logp"] = lp.gather(1, ids), tl + 4 * U32 * (fin(z.gather(1, ids)) + fin(lse))
    if dlogp is not None or dentropy is not None:
        zero = torch.zeros(x.shape[0], 1, dtype=F64)
        dl = d(dlogp).reshape(-1, 1) if dlogp is not None else zero
        if t is not None and dlogp is not None:
            dl = torch.where(skip[:, None], 0.0, torch.where(hit, dl, math.nan))
        de = d(dentropy).reshape(-1, 1) if dentropy is not None else zero
        flp = torch.where(p > 0, torch.where(torch.isfinite(lp), lp, 0.0), 0.0)
        g = -p * (dl + de * (flp + ent))
        ep = tl + 6 * U32 * (fin(z) + fin(lse)) + 8 * U32
        mag = dl.abs() + de.abs() * (flp.abs() + ent)
        tg = p * mag * (ep + 8 * U32) + p * de.abs() * (te + ep) + TINY * (mag + 130 * de.abs())
        if t is not None and dlogp is not None:
            one = torch.zeros_like(g).scatter_(1, at, 1.0) * hit
            g, tg = g + torch.where(one > 0, dl, 0.0), tg + one * 4 * U32 * torch.nan_to_num(dl).abs()
        dead = none | ((dl == 0) & (de == 0))
        g, tg = torch.where(dead, 0.0, g) * sc, torch.where(dead, 0.0, tg) * sc
        out["dlogits"] = g, rounding(torch.nan_to_num(g), dtype) + torch.nan_to_num(tg) + 2 * U32 * torch.nan_to_num(g).abs()
    return out, ids
