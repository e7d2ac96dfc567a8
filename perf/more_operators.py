"""What is timed of the operators around attention: the two ends of a model and what lies between its attention blocks.

  op "embed"       rows of a table by token, times a number; with `back`, that and the table's gradient, of which every row is written
  op "norm"        norms of whole rows, centred (layer norm) or not, weight and bias; with `back`, the forward and the backward pass, which
                   is given the inputs and works the statistics out again
  op "gated"       activation(x gate) * (x up), the first half of a gated MLP; with `back`, the forward and the backward pass, which is given
                   x and the weights and nothing that the forward pass computed
  op "log_probs"   logarithms of given tokens' probabilities, `entropy` and the `top` likeliest tokens of each row; with `back`, the gradient
                   of the logits too

Models are those of the traces: the encoder (768 values, 30522 tokens) and the decoder (4096 values, 16384 inside its MLP, 32000 tokens).
"""
import math

import torch

own = False

TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"fp32": 4, "fp16": 2, "bf16": 2}
EPS = 1e-6
IGNORE = -100


def _embed(**kw):
    return dict(dict(op="embed", dtype="bf16", batch=1, seq=1, vocab=32000, dim=4096, scale=1.0, ids64=False, back=False), **kw)


def _norm(**kw):
    return dict(dict(op="norm", dtype="bf16", weights="bf16", batch=1, seq=1, dim=4096, center=False, bias=False, back=False), **kw)


def _gated(**kw):
    return dict(dict(op="gated", dtype="bf16", tokens=1, dim=4096, inner=16384, act="silu", out_in=False, back=False), **kw)


def _log_probs(**kw):
    return dict(dict(op="log_probs", dtype="bf16", rows=1, vocab=32000, padded=0, tokens=True, entropy=False, top=0, scale=1.0, back=False), **kw)


def listed():
    return [
        # one new token of a few sequences
        _embed(name="embed_token", batch=8),
        # a training step of the decoder: 16 sequences of 2048 tokens, frequent tokens and rare ones, rows scaled by the root of their length
        _embed(name="embed_decoder_back", batch=16, seq=2048, scale=64.0, back=True),
        # a training step of the encoder, 32-bit weights, the ids that a tokenizer's loader hands over
        _embed(name="embed_encoder_back", dtype="fp32", batch=32, seq=512, vocab=30522, dim=768, ids64=True, back=True),
        # one new token of a few sequences
        _norm(name="norm_token", batch=4),
        # a layer of the decoder, forward
        _norm(name="norm_decoder", batch=16, seq=2048),
        # a training step of the encoder's layer norm: 32-bit weight and bias on half-precision activations
        _norm(name="norm_encoder_back", dtype="fp16", weights="fp32", batch=32, seq=512, dim=768, center=True, bias=True, back=True),
        # one new token of a few sequences: the decoder's weights are all there is to read
        _gated(name="gated_token", tokens=8),
        # a training step of the decoder's layer, four sequences of 2048 tokens
        _gated(name="gated_decoder_back", tokens=8192, back=True),
        # odd sizes, weights as a linear layer keeps them
        _gated(name="gated_odd_back", dtype="fp16", tokens=5001, dim=1000, inner=2744, act="gelu", out_in=True, back=True),
        # what a sampler asks for one new token of a few sequences: the 20 likeliest with their probabilities, and the entropy
        _log_probs(name="logp_token", rows=8, tokens=False, entropy=True, top=20),
        # the loss of a training step of the decoder and its gradient
        _log_probs(name="logp_decoder_back", rows=16 * 2048, back=True),
        # texts scored at a temperature, 32-bit logits of the encoder's vocabulary, padded columns masked
        _log_probs(name="logp_score", dtype="fp32", rows=1500, vocab=30522, padded=26, entropy=True, top=5, scale=1.25),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def _dim(rng, lo, hi):
    """A width: half of them whole hundreds of bytes, the others as they come."""
    n = _log(rng, lo, hi)
    return n if rng.random() < 0.4 else max(64, n // 64 * 64)


def draw(rng):
    op = rng.choice(["embed", "norm", "gated", "log_probs"])
    if op == "embed":
        dtype, dim, back = rng.choice(["fp32", "fp16", "bf16", "bf16"]), _dim(rng, 32, 8192), rng.random() < 0.6
        most = 32000 * 4096 * 2 // (dim * SIZE[dtype])
        vocab = _log(rng, 100, min(most, 131072))
        tokens = _log(rng, 1, min(most, 65536))
        batch = rng.choice([1, 2, 3, 5, 8, 16])
        return _embed(dtype=dtype, batch=batch, seq=max(1, tokens // batch), vocab=vocab, dim=dim, scale=rng.choice([1.0, 1.0, 0.5, math.sqrt(dim)]),
                      ids64=rng.random() < 0.5, back=back)
    if op == "norm":
        dtype, dim = rng.choice(["fp32", "fp16", "bf16", "bf16"]), _dim(rng, 32, 12288)
        back = rng.random() < 0.6
        most = 16 * 2048 * 4096 * 2 // (dim * SIZE[dtype]) // (2 if back else 1)
        center = rng.random() < 0.5
        batch = rng.choice([1, 2, 3, 4, 8])
        return _norm(dtype=dtype, weights=rng.choice([dtype, "fp32"]), batch=batch, seq=max(1, _log(rng, 1, most) // batch), dim=dim, center=center,
                     bias=center and rng.random() < 0.7, back=back)
    if op == "gated":
        dim, inner, back = _dim(rng, 64, 6144), _dim(rng, 64, 16384), rng.random() < 0.6
        most = 8192 * 4096 * 16384 // (dim * inner)
        return _gated(dtype=rng.choice(["fp16", "bf16", "bf16"]), tokens=rng.choice([_log(rng, 1, min(64, most)), _log(rng, 1, min(16384, most))]), dim=dim,
                      inner=inner, act=rng.choice(["silu", "silu", "gelu"]), out_in=rng.random() < 0.5, back=back)
    dtype, vocab = rng.choice(["fp32", "fp16", "bf16", "bf16"]), _log(rng, 50, 200000)
    back = rng.random() < 0.4
    most = 16 * 2048 * 32000 * 2 // (vocab * SIZE[dtype]) // (1 if back else 4)
    top = 0 if back else rng.choice([0, 1, 5, 20])
    tokens = back or not top or rng.random() < 0.6
    return _log_probs(dtype=dtype, rows=_log(rng, 1, min(most, 65536)), vocab=vocab, padded=rng.choice([0, 0, vocab // 20]), tokens=tokens,
                      entropy=rng.random() < 0.5, top=top, scale=rng.choice([1.0, 1.0, 1.25, 0.7]), back=back)


def work(case):
    e = SIZE[case["dtype"]]
    if case["op"] == "embed":
        tokens = case["batch"] * case["seq"]
        ids, values = tokens * (8 if case["ids64"] else 4), tokens * case["dim"]
        rows = min(tokens, case["vocab"]) * case["dim"] * e              # (table rows that are read, at most)
        if case["back"]:
            return {"bytes": ids + rows + 2 * values * e + case["vocab"] * case["dim"] * e, "flops": 2 * values}
        return {"bytes": ids + rows + values * e, "flops": values}
    if case["op"] == "norm":
        values = case["batch"] * case["seq"] * case["dim"]
        w = case["dim"] * SIZE[case["weights"]] * (2 if case["bias"] else 1)
        if case["back"]:                         # x, dy in; y, dx, the gradients of weight and bias out
            return {"bytes": 4 * values * e + 2 * w, "flops": 18 * values}
        return {"bytes": 2 * values * e + w, "flops": 6 * values}
    if case["op"] == "gated":
        m, k, n = case["tokens"], case["dim"], case["inner"]
        if case["back"]:                         # x, weights, dh in; h, dx, the weights' gradients out; two products forward, four back
            return {"bytes": (2 * m * k + 2 * m * n + 4 * k * n) * e, "flops": 12 * m * k * n}
        return {"bytes": (m * k + m * n + 2 * k * n) * e, "flops": 4 * m * k * n}
    r, v = case["rows"], case["vocab"]
    few = r * (8 * case["tokens"] + 4 + 4 * case["entropy"] + 12 * case["top"])
    return {"bytes": (2 if case["back"] else 1) * r * v * e + few, "flops": (8 if case["back"] else 5) * r * v}


# ---------------------------------------------------------------------------------------------------------- inputs
def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed * 1000003 + 29)

    def normal(*shape, dtype=torch.float32, scale=1.0):
        x = torch.randn(*shape, device="cuda", dtype=torch.float32 if math.prod(shape) < 1 << 28 else dtype, generator=g)
        return x.mul_(scale).to(dtype)

    dt = TYPES[case["dtype"]]
    st = dict(case=case)
    if case["op"] == "embed":
        b, s, v, d = (case[k] for k in ("batch", "seq", "vocab", "dim"))
        # the n-th most frequent token as often as 1 / (n + 2.7), tokens in no order
        u = torch.rand(b, s, device="cuda", dtype=torch.float64, generator=g)
        rank = (2.7 * ((v + 2.7) / 2.7) ** u - 2.7).long().clamp(0, v - 1)
        st["ids"] = torch.randperm(v, device="cuda", generator=g)[rank].to(torch.int64 if case["ids64"] else torch.int32)
        st["table"] = normal(v, d, dtype=dt, scale=0.02)
        if case["back"]:
            st["dout"] = normal(b, s, d, dtype=dt, scale=0.05)
        return st
    if case["op"] == "norm":
        b, s, d, wt = case["batch"], case["seq"], case["dim"], TYPES[case["weights"]]
        # a residual stream: rows of many sizes, off zero, a few places far larger than the others
        x = normal(b, s, d, dtype=dt, scale=1.3)
        x *= torch.exp(normal(b, s, 1)).to(dt)
        x += 0.3
        x[..., ::max(1, d // 3)] *= 20
        st["x"], st["weight"] = x, (1 + normal(d, scale=0.2)).to(wt)
        st["bias"] = normal(d, dtype=wt, scale=0.2) if case["bias"] else None
        if case["back"]:
            st["dy"] = normal(b, s, d, dtype=dt, scale=0.05)
        return st
    if case["op"] == "gated":
        m, k, n = case["tokens"], case["dim"], case["inner"]
        st["x"] = normal(m, k, dtype=dt)
        for name in ("gate", "up"):
            w = normal(n, k, dtype=dt, scale=1 / math.sqrt(k)) if case["out_in"] else normal(k, n, dtype=dt, scale=1 / math.sqrt(k))
            st[name] = w.t() if case["out_in"] else w
        if case["back"]:
            st["dh"] = normal(m, n, dtype=dt, scale=0.05)
        return st
    r, v = case["rows"], case["vocab"]
    x = normal(r, v, dtype=dt, scale=1.5)
    x += normal(v, scale=1.5).to(dt)                                     # what is likely everywhere
    live = v - case["padded"]
    t = torch.randint(0, live, (r,), device="cuda", generator=g)
    x.scatter_add_(1, t[:, None], normal(r, 1, scale=4.0).abs().to(dt))  # the model knows something
    x[:, live:] = -math.inf                                              # columns that no token has
    st["logits"], st["tokens"] = x, None
    if case["tokens"]:
        st["tokens"] = torch.where(torch.rand(r, device="cuda", generator=g) < 0.1, IGNORE, t)       # a prompt's tokens do not count
    if case["back"]:
        st["dlogp"] = normal(r, scale=1 / r)
        st["dentropy"] = normal(r, scale=0.1 / r) if case["entropy"] else None
    return st


# ---------------------------------------------------------------------------------------------------------- the plain forms
def _plain_embed(st):
    case, table, ids = st["case"], st["table"], st["ids"].long()
    out = {"out": (table[ids].float() * case["scale"]).to(table.dtype)}
    if case["back"]:
        sums = torch.zeros(table.shape, device="cuda", dtype=torch.float64)
        sums.index_add_(0, ids.flatten(), st["dout"].flatten(0, 1).double())
        out["dtable"] = (sums * case["scale"]).float().to(table.dtype)
    return out


def _plain_norm(st):
    case, x = st["case"], st["x"].float()
    w = st["weight"].float()
    c = x - x.double().mean(-1, keepdim=True).float() if case["center"] else x
    r = torch.rsqrt(c.square().mean(-1, keepdim=True) + EPS)
    n = c * r
    y = n * w
    if case["bias"]:
        y = y + st["bias"].float()
    out = {"y": y.to(st["x"].dtype)}
    if case["back"]:
        dy = st["dy"].float()
        u = dy * w
        dx = u - n * (u * n).mean(-1, keepdim=True)
        if case["center"]:
            dx = dx - u.mean(-1, keepdim=True)
        out["dx"] = (dx * r).to(st["x"].dtype)
        out["dweight"] = (dy * n).double().sum((0, 1)).to(st["weight"].dtype)
        if case["bias"]:
            out["dbias"] = dy.double().sum((0, 1)).to(st["bias"].dtype)
    return out


def _plain_gated(st):
    case, x, wg, wu = st["case"], st["x"].float(), st["gate"].float(), st["up"].float()
    dt = st["x"].dtype
    g, u = x @ wg, x @ wu
    if case["act"] == "silu":
        s = 1 / (1 + torch.exp(-g))
        a, slope = g * s, s * (1 + g * (1 - s))
    else:
        s = 0.5 * (1 + torch.erf(g * math.sqrt(0.5)))
        a, slope = g * s, s + g * torch.exp(-0.5 * g * g) * (1 / math.sqrt(2 * math.pi))
    out = {"h": (a * u).to(dt)}
    if case["back"]:
        dh = st["dh"].float()
        dg, du = dh * u * slope, dh * a
        del g, u, s, a, slope
        out["dx"] = (dg @ wg.t() + du @ wu.t()).to(dt)
        out["dgate"], out["dup"] = (x.t() @ dg).to(dt), (x.t() @ du).to(dt)
    return out


def _plain_log_probs(st):
    case, scale = st["case"], st["case"]["scale"]
    x = st["logits"].float()
    z = x * scale
    top = z.amax(-1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(-1, keepdim=True)
    lse = top + torch.log(total)
    out = {"lse": lse[:, 0]}
    known = t = None
    if case["tokens"]:
        known = st["tokens"] != IGNORE
        t = torch.where(known, st["tokens"], 0)[:, None]
        out["logp"] = torch.where(known, (z.gather(1, t) - lse)[:, 0], 0.0)
    if case["entropy"]:
        out["entropy"] = -(e / total * torch.where(e > 0, z - lse, 0.0)).sum(-1)
    if case["top"]:
        best = torch.sort(x, dim=-1, descending=True, stable=True)[1][:, :case["top"]]
        out["top_ids"], out["top_logp"] = best, z.gather(1, best) - lse
    if case["back"]:
        p = e.div_(total)
        dl = torch.where(known, st["dlogp"], 0.0)[:, None]
        dz = p * -dl
        if case["entropy"]:
            dz -= p * (torch.where(p > 0, z - lse, 0.0) + out["entropy"][:, None]) * st["dentropy"][:, None]
        dz.scatter_add_(1, t, dl)
        out["dlogits"] = (dz * scale).to(st["logits"].dtype)
    return out


# ---------------------------------------------------------------------------------------------------------- one pass
def run(st):
    case = st["case"]
    if not own:
        return {"embed": _plain_embed, "norm": _plain_norm, "gated": _plain_gated, "log_probs": _plain_log_probs}[case["op"]](st)
    from paper_2310_09443_amd import ops
    if case["op"] == "embed":
        out = dict(out=ops.g10_embed(st["ids"], st["table"], scale=case["scale"]))
        if case["back"]:
            out["dtable"] = ops.g10_embed_backward(st["dout"], st["ids"], case["vocab"], scale=case["scale"])
        return out
    if case["op"] == "norm":
        args = dict(weight=st["weight"], bias=st["bias"], eps=EPS, center=case["center"])
        out = dict(y=ops.g10_norm(st["x"], **args))
        if case["back"]:
            out["dx"], out["dweight"], dbias = ops.g10_norm_backward(st["dy"], st["x"], **args)
            if case["bias"]:
                out["dbias"] = dbias
        return out
    if case["op"] == "gated":
        out = dict(h=ops.g10_gated(st["x"], st["gate"], st["up"], act=case["act"]))
        if case["back"]:
            out["dx"], out["dgate"], out["dup"] = ops.g10_gated_backward(st["dh"], st["x"], st["gate"], st["up"], act=case["act"])
        return out
    logp, lse, entropy, top_logp, top_ids = ops.g10_log_probs(st["logits"], st["tokens"], scale=case["scale"], entropy=case["entropy"], top=case["top"],
                                                              ignore=IGNORE)
    out = dict(lse=lse)
    if case["tokens"]:
        out["logp"] = logp
    if case["entropy"]:
        out["entropy"] = entropy
    if case["top"]:
        out.update(top_ids=top_ids, top_logp=top_logp)
    if case["back"]:
        out["dlogits"] = ops.g10_log_probs_backward(st["dlogp"], st["logits"], st["tokens"], lse, scale=case["scale"], ignore=IGNORE,
                                                    dentropy=st["dentropy"], entropy=entropy)
    return out


# ---------------------------------------------------------------------------------------------------------- in 64 bits
def _exact_embed(st):
    case, ids = st["case"], st["ids"].flatten().long()
    table = st["table"].double()
    out = {"out": torch.index_select(table, 0, ids).view(case["batch"], case["seq"], -1) * case["scale"]}
    if case["back"]:
        del table
        # tokens in order, running sums, and what they grow by over each token's run
        order = torch.argsort(ids)
        runs = torch.cumsum(st["dout"].flatten(0, 1)[order].double(), 0)
        runs = torch.cat([torch.zeros_like(runs[:1]), runs])
        ends = torch.searchsorted(ids[order], torch.arange(case["vocab"] + 1, device="cuda"))
        out["dtable"] = torch.diff(runs[ends], dim=0) * case["scale"]
    return out


def _exact_norm(st):
    case, x, d = st["case"], st["x"].double(), st["case"]["dim"]
    w = st["weight"].double()
    mean = x.sum(-1, keepdim=True) / d if case["center"] else 0.0
    size = torch.sqrt((x - mean).pow(2).sum(-1, keepdim=True) / d + EPS)
    y = (x - mean) / size * w
    out = {"y": y + st["bias"].double() if case["bias"] else y}
    if case["back"]:
        dy = st["dy"].double()
        gw = dy * w
        # each value's own share, less the shares through the size and the mean of the whole row
        dx = gw / size - (x - mean) * ((gw * (x - mean)).sum(-1, keepdim=True) / (d * size ** 3))
        out["dx"] = dx - gw.sum(-1, keepdim=True) / (d * size) if case["center"] else dx
        out["dweight"] = ((x - mean) / size * dy).flatten(0, 1).sum(0)
        if case["bias"]:
            out["dbias"] = dy.flatten(0, 1).sum(0)
    return out


def _exact_gated(st):
    x, wg, wu = (st[n].double() for n in ("x", "gate", "up"))
    g, u = torch.mm(x, wg), torch.mm(x, wu)
    phi = torch.sigmoid(g) if st["case"]["act"] == "silu" else torch.special.ndtr(g)
    out = {"h": g * phi * u}
    if st["case"]["back"]:
        density = phi * (1 - phi) if st["case"]["act"] == "silu" else torch.exp(-g.pow(2) / 2) / math.sqrt(2 * math.pi)
        dh = st["dh"].double()
        dup = dh * g * phi
        dgate = dh * u * (phi + g * density)
        out["dx"] = torch.mm(dup, wu.T) + torch.mm(dgate, wg.T)
        out["dgate"], out["dup"] = torch.mm(dgate.T, x).T, torch.mm(dup.T, x).T
    return out


def _exact_log_probs(st):
    case = st["case"]
    parts = {}
    step = max(1, (1 << 28) // case["vocab"])
    for a in range(0, case["rows"], step):                               # some rows at a time: 64 bits of all of them are 8 GB
        at = slice(a, a + step)
        z = st["logits"][at].double() * case["scale"]
        l = torch.logsumexp(z, -1, keepdim=True)
        logs = z - l
        p = logs.exp()
        out = {"lse": l[:, 0]}
        if case["entropy"]:
            out["entropy"] = torch.special.entr(p).sum(-1)
        if case["top"]:
            out["top_logp"] = torch.topk(logs, case["top"], -1)[0]
        if case["tokens"]:
            t, skip = st["tokens"][at], st["tokens"][at] == IGNORE
            t = t.masked_fill(skip, 0)
            out["logp"] = logs[torch.arange(len(t), device="cuda"), t].masked_fill(skip, 0.0)
        if case["back"]:
            dl = st["dlogp"][at].double().masked_fill(skip, 0.0)
            dz = -p * dl[:, None]
            dz[torch.arange(len(t), device="cuda"), t] += dl
            if case["entropy"]:
                dz += (torch.special.entr(p) - p * out["entropy"][:, None]) * st["dentropy"][at].double()[:, None]
            out["dlogits"] = dz * case["scale"]
        for n, x in out.items():
            parts.setdefault(n, []).append(x)
    out = {n: torch.cat(x) for n, x in parts.items()}
    if case["top"]:
        out["top_ids"] = None
    return out


def exact(case, seed):
    st = prepare(case, seed)
    return {"embed": _exact_embed, "norm": _exact_norm, "gated": _exact_gated, "log_probs": _exact_log_probs}[case["op"]](st)
