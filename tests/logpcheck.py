"""Log probabilities in 64 bits on the CPU, with bounds that go by distances from the row's largest logit and by the additions that a thread makes: a row
whose logits have an offset in common, or lie at the type's end, is as exact as one around zero.  (lse alone is a place, not a distance: it is
rounded to 32 bits where it lies.)"""
import math

import torch

from opscheck import F64, U32, assert_near, d, rounding  # noqa: F401

F32 = torch.finfo(torch.float32)


def additions(v):
    """Additions behind a row's sum, one behind the other: a wavefront takes rows of up to 512 pieces of 16 bytes, 4096 values, and 256 threads or more take
    longer ones; then 6 steps in the wavefront, up to 16 wavefronts and 16 parts."""
    return max(64, v / 256) + 16 + 6 + 16 + 16


def log_probs(logits, tokens, scale, ignore=-100, top=0, dlogp=None, dentropy=None, near=0.0):
    """{name: (value, tolerance)}, and the ids of the top.  near: the gradient may take a row's probabilities from lse as it is, rounded, up to this size."""
    dtype, v, sc = logits.dtype, logits.shape[-1], float(torch.tensor(scale, dtype=torch.float32))
    x = d(logits).reshape(-1, v)
    m = x.amax(-1, keepdim=True)
    none = m == -math.inf
    m0 = torch.where(none, 0.0, m)
    dist = (x - m0) * sc
    fin = torch.where(x == -math.inf, 0.0, dist)
    e = torch.where(x == -math.inf, 0.0, torch.exp(dist))
    s = torch.where(none, 1.0, e.sum(-1, keepdim=True))
    ls, p = torch.log(s), e / s
    lp = torch.where(none, -math.inf, dist - ls)
    far = (p * fin.abs()).sum(-1, keepdim=True)
    # The logarithm of the sum.  An exponential's argument is off by what scale in powers of two (2 roundings), its difference and the moves of the
    # maximum leave, 6 roundings of the distance; itself by 2; a thread's sum is scaled where its maximum moves, 3 roundings for 4 values or more: 2 for
    # each addition.  The maximum in powers of two is rounded by up to 4, which the logarithm carries and the difference takes out again.
    es = (2 * additions(v) + 40 + 6 * far + 2 * ls) * U32
    lse = torch.where(none, -math.inf, m0 * sc + ls)
    flse = torch.where(none, 0.0, m0 * sc + ls)
    tlse = es + 6 * U32 * ((m0 * sc).abs() + flse.abs())
    over = flse.abs() > F32.max                                      # (rounds to an infinity)
    out = {"lse": (torch.where(over, flse.sign() * math.inf, lse)[:, 0], tlse[:, 0])}
    te = 2 * es * (1 + far + ls + (2 * U32 * (m0 * sc).abs()).clamp(max=4))     # (distances there have the maximum's rounding in them)
    ent = torch.where(none, 0.0, ls + far)
    out["entropy"] = ent[:, 0], te[:, 0]

    def error(dist):                                                  # of a place's logarithm
        return es + U32 * (6 * torch.where(torch.isfinite(dist), dist, 0.0).abs() + 4 * ls + 40)

    def as_held(y):                                                   # (a distance beyond 32 bits is an infinity)
        return torch.where(y < -F32.max, -math.inf, y)
    hit = at = None
    if tokens is not None:
        t = tokens.reshape(-1).cpu().long()
        skip, hit = (t == ignore)[:, None], ((t >= 0) & (t < v) & (t != ignore))[:, None]
        at = t.clamp(0, v - 1)[:, None]
        out["logp"] = (torch.where(skip, 0.0, torch.where(hit, as_held(lp.gather(1, at)), math.nan))[:, 0], torch.where(hit, error(dist.gather(1, at)), 0.0)[:, 0])
    ids = None
    if top:
        ids = torch.sort(x, dim=-1, descending=True, stable=True)[1][:, :top]
        out["top_logp"] = as_held(lp.gather(1, ids)), error(dist.gather(1, ids))
    if dlogp is not None or dentropy is not None:
        zero = torch.zeros(x.shape[0], 1, dtype=F64)
        dl = d(dlogp).reshape(-1, 1) if dlogp is not None else zero
        de = d(dentropy).reshape(-1, 1) if dentropy is not None else zero
        if dlogp is not None:                                         # (a share of nothing is nothing, whatever the token)
            dl = torch.where(skip, 0.0, torch.where(hit | (dl == 0), dl, math.nan))
        flp = torch.where(p > 0, lp, 0.0)
        ep = error(fin) + torch.where(flse.abs() < near, 6 * U32 * ((m0 * sc).abs() + flse.abs()), 0.0) + 4 * U32 * flp.abs() + 8 * U32
        mag = dl.abs() + de.abs() * (flp.abs() + ent)
        g = -p * (dl + de * (flp + ent))
        tg = p * mag * (ep + 8 * U32) + p * de.abs() * (te + ep) + F32.tiny * (mag + 130 * de.abs())
        if dlogp is not None:
            one = torch.zeros_like(g).scatter_(1, at, 1.0) * hit
            g, tg = g + torch.where(one > 0, dl, 0.0), tg + one * 4 * U32 * torch.nan_to_num(dl).abs()
        dead = none | ((dl == 0) & (de == 0))
        g, tg = torch.where(dead, 0.0, g) * sc, torch.where(dead, 0.0, tg) * sc
        out["dlogits"] = g, rounding(torch.nan_to_num(g), dtype) + torch.nan_to_num(tg) + 2 * U32 * torch.nan_to_num(g).abs()
    return out, ids


def check(got, want):
    """got: name to tensor; want: as above."""
    for n, (y, t) in want.items():
        if n in got:
            assert_near(got[n].reshape(y.shape), y, t, n)
