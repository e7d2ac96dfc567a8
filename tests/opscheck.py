"""The operators of include/g10_ops.h in 64 bits on the CPU, from their formulas, and how far an implementation that rounds where
the header says may be from them.  u(t) is half a step of a type: a rounding is off by at most u |value|."""
import math

import torch

F64 = torch.float64


def u(dtype):
    return torch.finfo(dtype).eps / 2


U32 = u(torch.float32)


def rounding(x, dtype):
    """How far one rounding takes x: u |x|, below the type's smallest normal number half the distance of its numbers there."""
    return (u(dtype) * x.abs()).clamp(min=torch.finfo(dtype).tiny * u(dtype))


def d(t):
    return None if t is None else t.detach().cpu().to(F64)


# ---------------------------------------------------------------------------------------------------- norm and rotation
def turn(x, table, positions, interleaved, back=False):
    rot = table.shape[1]
    t = table[positions.long()][..., None, :]                         # [..., token, 1, rot]
    c, s = t[..., :rot // 2], t[..., rot // 2:]
    if back:
        s = -s
    i = torch.arange(rot // 2)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
    y = x.clone()
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    size = x.abs().clone()                                            # sum of the magnitudes that meet in a value
    size[..., a] = (x[..., a] * c).abs() + (x[..., b] * s).abs()
    size[..., b] = (x[..., b] * c).abs() + (x[..., a] * s).abs()
    return y, size


def rope(x, w, table, positions, eps, interleaved, dtype):
    """(y, tolerance)"""
    x, table = d(x), d(table)
    w = torch.ones(x.shape[-1], dtype=F64) if w is None else d(w)
    n = x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * w
    y, size = turn(n, table, positions.cpu(), interleaved)
    # the sum of squares (dim additions, each off by u), half of which reaches the root; root, division, 3 products, 1 sum
    return y, rounding(y, dtype) + (x.shape[-1] / 2 + 8) * U32 * size


def rope_backward(dy, x, w, table, positions, eps, interleaved, dtype):
    """dx, dw and their tolerances"""
    dim = x.shape[-1]
    dy, x, table = d(dy), d(x), d(table)
    w = torch.ones(dim, dtype=F64) if w is None else d(w)
    r = 1 / (x.square().mean(-1, keepdim=True) + eps).sqrt()
    n = x * r
    g, size = turn(dy, table, positions.cpu(), interleaved, back=True)
    dot = (g * w * n).mean(-1, keepdim=True)
    dx = r * (g * w - n * dot)
    mag = r * (size * w.abs() + n.abs() * (size * w.abs() * n.abs()).mean(-1, keepdim=True))
    lead = tuple(range(x.dim() - 1))
    dw, wmag = (g * n).sum(lead), (size * n.abs()).sum(lead)
    rows = x.numel() // dim
    return dx, rounding(dx, dtype) + (2 * dim + 16) * U32 * mag, dw, wmag * (dim / 2 + 16 + min(rows, 256)) * U32


# ------------------------------------------------------------------------------------------------------------ attention
def visible(nq, nk, causal, window, sinks):
    p = torch.arange(nq)[:, None] + nk - nq
    j = torch.arange(nk)[None]
    near = torch.ones(nq, nk, dtype=torch.bool)
    if window:
        near = ((p - j < window) if causal else ((p - j).abs() < window)) | (j < sinks)
    return near & (j <= p) if causal else near


def attention_one(q, k, v, do, causal, window, sinks, scale, dtype):
    """One sequence, one group of heads: q, do [heads, nq, dim], k, v [nk, dim].  {name: (value, tolerance)}."""
    q, k, v, do = d(q), d(k), d(v), d(do)
    nq, nk, dim, e = q.shape[1], k.shape[0], q.shape[2], u(dtype)
    seen = visible(nq, nk, causal, window, sinks)
    s = (q @ k.T) * scale
    s = s.masked_fill(~seen, -math.inf)
    top = s.amax(-1, keepdim=True) if nk else torch.full((*q.shape[:2], 1), -math.inf, dtype=F64)
    x = torch.exp(s - torch.where(top == -math.inf, 0.0, top))
    l = x.sum(-1, keepdim=True)
    P = x / torch.where(l == 0, 1.0, l)
    o = P @ v
    lse = torch.where(l == 0, -math.inf, top + torch.log(l))[..., 0]
    # a score is a sum of dim products in 32 bits, scaled once; exponentials are good to 4 u, their sum of nk terms in any order
    ds = (dim + 4) * U32 * ((q.abs() @ k.abs().T) * scale).amax(-1, keepdim=True) if nk else torch.zeros(*q.shape[:2], 1, dtype=F64)
    ep = 2 * ds + (8 + nk) * U32 + U32 * torch.where(torch.isfinite(top), top, 0.0).abs() * 4
    A = P @ v.abs()
    least = torch.finfo(torch.float32).tiny                           # an exponential below the smallest normal number may be zero
    to = rounding(o, dtype) + (e + ep) * A + nk * U32 * A + least * v.abs().sum(0)       # one rounding of o, one of each P
    out = {"o": (o, to), "lse": (lse, ep[..., 0] + 8 * U32 * (1 + torch.where(torch.isfinite(lse), lse, 0.0).abs()))}
    if do is None:
        return out
    dP = do @ v.T
    delta = (do * o).sum(-1, keepdim=True)
    dS = P * (dP - delta) * scale
    # delta is taken from the rounded o
    tdelta = (do.abs() * (to + dim * U32 * o.abs())).sum(-1, keepdim=True)
    mag = do.abs() @ v.abs().T
    tiny = (2.0 ** -25 * do.abs().max() / 4 * scale if dtype == torch.float16 and do.numel() else 0.0)   # fp16's smallest numbers, lifted
    tS = (e + ep) * dS.abs() + P * scale * (tdelta + (dim + 4) * U32 * (mag + delta.abs()) * (1 + ep)) + tiny + least * scale * (mag + delta.abs())
    tP = (e + ep) * P + least + (2.0 ** -37 if dtype == torch.float16 else 0.0)
    n = nq * q.shape[0]
    dq, dk, dv = dS @ k, (dS.transpose(1, 2) @ q).sum(0), (P.transpose(1, 2) @ do).sum(0)
    out["dq"] = dq, rounding(dq, dtype) + tS @ k.abs() + nk * U32 * (dS.abs() @ k.abs())
    out["dk"] = dk, rounding(dk, dtype) + (tS.transpose(1, 2) @ q.abs()).sum(0) + n * U32 * (dS.abs().transpose(1, 2) @ q.abs()).sum(0)
    out["dv"] = dv, rounding(dv, dtype) + (tP.transpose(1, 2) @ do.abs()).sum(0) + n * U32 * (P.transpose(1, 2) @ do.abs()).sum(0)
    return out


def attention(q, k, v, do, causal, window, sinks, scale=None, q_start=None, k_start=None, k_len=None):
    """{name: (value, tolerance)} with the layouts of ops.g10_attention."""
    heads, kv, dim = q.shape[-2], k.shape[-2], q.shape[-1]
    scale = dim ** -0.5 if scale is None else scale
    dtype, packed, group = q.dtype, q_start is not None, heads // kv
    shapes = {"o": q.shape, "lse": (heads, q.shape[0]) if packed else (q.shape[0], heads, q.shape[1])}
    if do is not None:
        shapes.update(dq=q.shape, dk=k.shape, dv=v.shape)
    out = {n: (torch.zeros(s, dtype=F64), torch.zeros(s, dtype=F64)) for n, s in shapes.items()}
    batch = len(q_start) - 1 if packed else q.shape[0]
    for b in range(batch):
        if packed:
            qr, kr = slice(int(q_start[b]), int(q_start[b + 1])), slice(int(k_start[b]), int(k_start[b + 1]))
            cut = {"q": (lambda t: t[qr]), "k": (lambda t: t[kr])}
        else:
            nk = int(k_len[b]) if k_len is not None else k.shape[1]
            cut = {"q": (lambda t: t[b]), "k": (lambda t: t[b, :nk])}
        for h in range(kv):
            hs = slice(h * group, (h + 1) * group)
            Q, dO = cut["q"](q)[:, hs].transpose(0, 1), cut["q"](do)[:, hs].transpose(0, 1) if do is not None else None
            got = attention_one(Q, cut["k"](k)[:, h], cut["k"](v)[:, h], dO, causal, window, sinks, scale, dtype)
            for n, (x, t) in got.items():
                for dst, src in zip(out[n], (x, t)):
                    if n == "lse":
                        (dst[hs, qr] if packed else dst[b, hs])[:] = src
                    elif n in ("o", "dq"):
                        cut["q"](dst)[:, hs] = src.transpose(0, 1)
                    else:
                        cut["k"](dst)[:, h] = src
    return out


def assert_near(got, want, tol, what=""):
    got = d(got)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    off = torch.where(same, 0.0, (got - want).abs())
    bad = ~(off <= tol + 1e-300)
    if bad.any():
        i = torch.where(bad, torch.nan_to_num(off / (tol + 1e-300), nan=1e9, posinf=1e9), 0.0).argmax()
        at = [int(x) for x in torch.unravel_index(i, got.shape)]
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} values off; at {at}: got {got.reshape(-1)[i]:.9g}, want "
                             f"{want.reshape(-1)[i]:.9g}, tolerance {tol.expand_as(want).reshape(-1)[i]:.3g}")


# ---------------------------------------------------------------------------------------------------------------- AdamW
def adamw(p, g, m, v, step, lr, b1, b2, eps, decay, coef=1.0):
    """p, m, v after a step, and the magnitudes that their roundings go by."""
    p, g, m, v = d(p), d(g) * coef, d(m), d(v)
    m1 = b1 * m + (1 - b1) * g
    v1 = b2 * v + (1 - b2) * g * g
    move = lr / (1 - b1 ** step) * m1 / ((v1 / (1 - b2 ** step)).sqrt() + eps)
    mm = (b1 * m).abs() + ((1 - b1) * g).abs()
    # m: two constants, two products, a sum and the coefficient; the move: m's share, a root, five more operations
    tm = 6 * U32 * mm
    spread = torch.where(m1 != 0, tm / m1.abs(), 0.0)
    tp = 12 * U32 * (p.abs() + move.abs()) + move.abs() * spread
    return (p * (1 - lr * decay) - move, tp), (m1, tm), (v1, 8 * U32 * v1)
