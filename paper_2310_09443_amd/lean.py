"""A decoder whose training step leaves the planner less to move, with the operators of `ops` together as they are used.

    python -m paper_2310_09443_amd.lean              # trains a small decoder, lets it continue a text, plans its big sister's step

`Decoder` is the decoder of the benchmark's fourth workload in small: norms of queries and keys with the rotation in one pass,
attention with a window and sinks, weights in bfloat16 beside 32-bit masters, one AdamW a layer with its moments in 8 bits.
(One a layer and not one for all: a launch needs what it works on in GPU memory at once, and what no launch needs the planner
may move.)  `decoder48_lean` is that workload's trace with these operators in the place of the ones that keep scores and 32-bit
moments; planning both says what they save.
"""
from __future__ import annotations

import math

import numpy as np

from . import traces


class Decoder:
    """`layers` blocks of `dim` values: attention over `heads` heads of 64 on `kv_heads`, a gated MLP of `inner` values."""

    HEAD = 64

    def __init__(self, vocab=256, dim=256, layers=2, heads=4, kv_heads=2, inner=512, window=64, sinks=4, max_len=1024, seed=0, lr=3e-3,
                 state_bits=8, device="cuda"):
        import torch
        from . import ops
        self.ops, self.torch = ops, torch
        self.dim, self.heads, self.kv, self.window, self.sinks, self.device = dim, heads, kv_heads, window, sinks, device
        gen = torch.Generator().manual_seed(seed)
        D = self.HEAD

        def weight(*shape, std=None):
            if std == 0:
                return torch.ones(shape)
            return torch.randn(shape, generator=gen) * (std or 1 / math.sqrt(shape[0]))

        groups = [dict(embed=weight(vocab, dim, std=0.02), out_norm=weight(dim, std=0), head=weight(dim, vocab))]
        for _ in range(layers):
            groups.append(dict(norm1=weight(dim, std=0), wqkv=weight(dim, (heads + 2 * kv_heads) * D), q_norm=weight(D, std=0), k_norm=weight(D, std=0),
                               wo=weight(heads * D, dim), norm2=weight(dim, std=0), gate=weight(dim, inner), up=weight(dim, inner), down=weight(inner, dim)))
        self.layers, self.opts = [], []
        for g in groups:
            masters = [t.to(device) for t in g.values()]
            copies = [t.to(torch.bfloat16).requires_grad_() for t in masters]        # what the passes read, refreshed by the update
            self.layers.append(dict(zip(g, copies)))
            self.opts.append(ops.AdamW(masters, lr=lr, weight_decay=0.0, state_bits=state_bits, copies=[c.detach() for c in copies]))
        self.table = ops.rope_table(max_len, D, device=device)

    def _norm(self, x, w):
        f = x.float()
        return (f * self.torch.rsqrt(f.square().mean(-1, keepdim=True) + 1e-6)).to(x.dtype) * w

    def _qkv(self, w, x):
        qkv = (self._norm(x, w["norm1"]) @ w["wqkv"]).unflatten(-1, (-1, self.HEAD))
        return qkv[:, :, :self.heads], qkv[:, :, self.heads:self.heads + self.kv], qkv[:, :, self.heads + self.kv:]

    def _mlp(self, w, x):
        n = self._norm(x, w["norm2"])
        return x + (self.torch.nn.functional.silu(n @ w["gate"]) * (n @ w["up"])) @ w["down"]

    def logits(self, ids):
        """[batch, token] -> [batch, token, vocab], differentiable."""
        torch, ops, top = self.torch, self.ops, self.layers[0]
        pos = torch.arange(ids.shape[1], device=self.device, dtype=torch.int32).expand(ids.shape)
        x = top["embed"][ids]
        for w in self.layers[1:]:
            q, k, v = self._qkv(w, x)
            q, k = ops.norm_rope(q, k, self.table, pos, w["q_norm"], w["k_norm"])
            o = ops.attention(q, k, v, window=self.window, sinks=self.sinks)
            x = self._mlp(w, x + o.flatten(2) @ w["wo"])
        return self._norm(x, top["out_norm"]) @ top["head"]

    def step(self, ids, max_norm=1.0):
        """One training step on [batch, token + 1]; returns (loss, norm of the gradients), device tensors."""
        torch = self.torch
        for w in self.layers:
            for t in w.values():
                t.grad = None
        loss = torch.nn.functional.cross_entropy(self.logits(ids[:, :-1]).float().flatten(0, 1), ids[:, 1:].flatten())
        loss.backward()
        grads = [[t.grad for t in w.values()] for w in self.layers]
        norm = torch.stack([o.grad_norm(g) for o, g in zip(self.opts, grads)]).square().sum().sqrt()
        coefficient = (max_norm / (norm + 1e-6)).clamp(max=1.0)
        for o, g in zip(self.opts, grads):
            o.step(g, coefficient=coefficient)
        return loss.detach(), norm

    def continue_text(self, ids, n):
        """`n` more tokens, the likeliest each time, one by one on caches of keys and values: [batch, token + n]."""
        torch, ops, top = self.torch, self.ops, self.layers[0]
        with torch.no_grad():
            b, s = ids.shape
            room = s + n
            caches = [[torch.zeros(b, room, self.kv, self.HEAD, dtype=torch.bfloat16, device=self.device) for _ in range(2)] for _ in self.layers[1:]]
            at, new = 0, ids
            for _ in range(n):
                m = new.shape[1]
                pos = torch.arange(at, at + m, device=self.device, dtype=torch.int32).expand(b, m)
                k_len = torch.full((b,), at + m, dtype=torch.int32, device=self.device)
                x = top["embed"][new]
                for w, (ck, cv) in zip(self.layers[1:], caches):
                    q, k, v = self._qkv(w, x)
                    q, k = ops.g10_norm_rope(q, k, self.table, pos, w["q_norm"], w["k_norm"])
                    ck[:, at:at + m], cv[:, at:at + m] = k, v
                    o, _ = ops.g10_attention(q, ck, cv, window=self.window, sinks=self.sinks, k_len=k_len)
                    x = self._mlp(w, x + o.flatten(2) @ w["wo"])
                at += m
                new = (self._norm(x[:, -1:], top["out_norm"]) @ top["head"]).argmax(-1)
                ids = torch.cat([ids, new], 1)
        return ids

    def close(self):
        for o in self.opts:
            o.close()


# Microseconds of the operators on an MI355X at the sizes of `decoder48_lean`; the update is bound by its bytes: 16 an element (master
# 4 + 4, gradient 2, moments 1 + 1 twice, copy 2) and the scales.
ROPE_US, ROPE_BACK_US, ATTENTION_US, ATTENTION_BACK_US = 210, 327, 677, 2470
ADAMW_BYTES, ADAMW_BPUS = 16 + 16 / 256, 5.2e6


def decoder48_lean(seed: int = 0x67100004) -> traces.Workload:
    """The 48-layer decoder of `traces.decoder48` (same sizes, same weights) with the operators of `ops`: per layer one kernel for the
    norms and the rotation, one for attention (kept for its backward pass: q, k, v, the output and one number a query and head), and
    one AdamW that reads masters, gradients and 8-bit moments and writes the working copies.  The durations of the operators are
    those measured on an MI355X at these sizes; the others are drawn as there."""
    Bt, S, H, NH, L, FF, V = 16, 2048, 4096, 32, 48, 16384, 32000
    esz, wsz = 2, 2
    rows = Bt * S
    g = traces._Graph(tmp_seed=seed, fwd_tmps=2, bwd_tmps=2, opt_tmps=2)
    us, back_us = {}, {}                      # an operator's kernel -> its duration; the gradient that its backward kernel begins with -> that one's
    ids = g.tensor(rows * 8)
    emb = g.weight(V * H * wsz)
    layer_weights = [[emb]]
    x = g.tensor(rows * H * esz)
    g.op([], [emb], [x], extra=[ids])
    rope = g.tensor(S * (H // NH) * 4, True)
    for _ in range(L):
        first = len(g.weights)
        h = traces._norm(g, x, H, rows, esz, wsz, affine_bias=False)
        wq, wk, wv = (g.weight(H * H * wsz) for _ in range(3))
        q, k, v = (g.tensor(rows * H * esz) for _ in range(3))
        for w, o in ((wq, q), (wk, k), (wv, v)):
            g.op([h], [w], [o], ws_bytes=32 << 20)
        qr, kr = g.tensor(rows * H * esz), g.tensor(rows * H * esz)
        norms = [g.weight(H // NH * wsz) for _ in range(2)]
        us[len(g.kernels)] = ROPE_US
        g.op([q, k], [], [qr, kr], saved=[q, k, rope] + norms + [g.grad_of(w) for w in norms], extra=[rope] + norms)
        back_us[g.grad_of(qr)] = ROPE_BACK_US
        ctx, lse = g.tensor(rows * H * esz), g.tensor(Bt * NH * S * 4)
        us[len(g.kernels)] = ATTENTION_US
        g.op([qr, kr, v], [], [ctx], saved=[qr, kr, v, ctx, lse], extra=[lse])
        back_us[g.grad_of(ctx)] = ATTENTION_BACK_US
        wo = g.weight(H * H * wsz)
        o = g.tensor(rows * H * esz)
        g.op([ctx], [wo], [o], ws_bytes=32 << 20)
        x1 = g.tensor(rows * H * esz)
        g.op([o, x], [], [x1], saved=[])
        h2 = traces._norm(g, x1, H, rows, esz, wsz, affine_bias=False)
        wg, wu, wd = g.weight(H * FF * wsz), g.weight(H * FF * wsz), g.weight(FF * H * wsz)
        gt, up = g.tensor(rows * FF * esz), g.tensor(rows * FF * esz)
        g.op([h2], [wg], [gt], ws_bytes=32 << 20)
        g.op([h2], [wu], [up], ws_bytes=32 << 20)
        act = g.tensor(rows * FF * esz)
        g.op([gt, up], [], [act])
        dn = g.tensor(rows * H * esz)
        g.op([act], [wd], [dn], ws_bytes=32 << 20)
        x = g.tensor(rows * H * esz)
        g.op([dn, x1], [], [x], saved=[])
        layer_weights.append(g.weights[first:])
    first = len(g.weights)
    hN = traces._norm(g, x, H, rows, esz, wsz, affine_bias=False)
    lm = g.weight(H * V * wsz)
    logits = g.tensor(rows * V * esz)
    g.op([hN], [lm], [logits], ws_bytes=32 << 20)
    layer_weights.append(g.weights[first:])
    labels, loss = g.tensor(rows * 8), g.tensor(4)
    g.op([logits], [], [loss], saved=[logits], extra=[labels])
    before = len(g.kernels)
    g.backward(split_weight_grads=True)
    for i in range(before, len(g.kernels)):
        if g.kernels[i][0] in back_us:
            us[i] = back_us[g.kernels[i][0]]
    g.phase = "opt"
    for ws in layer_weights:
        uses, n = [], 0
        for w in ws:
            e = g.sizes[w] // wsz
            n += e
            uses += [w] + ([g.grad[w]] if w in g.grad else []) + [g.tensor(4 * e, True)] + [g.tensor(e + 4 * -(-e // 256), True) for _ in range(2)]
        us[len(g.kernels)] = max(5, round(n * ADAMW_BYTES / ADAMW_BPUS))
        g.kernel(uses)
    dur = traces.rand_lognormal_ns(seed, 1, len(g.kernels), 200_000.0, 1.2)
    for i, d in us.items():
        dur[i] = d * 1000
    return traces.Workload(g.finish("decoder48_lean", np.asarray(dur)), cap_frac=0.30, meta=dict(batch=Bt, seq=S, hidden=H, layers=L))


def compare_plans(gpu_bytes=288 * 10**9, host_bytes=512 << 30):
    """Both traces planned for one machine: [(name, peak bytes, peak bytes that the plan leaves, migrations,
    bytes moved out and in, iteration ns, stall ns)]."""
    from . import binding
    out = []
    for w in (traces.decoder48(), decoder48_lean()):
        h = binding.g10_vitality(binding.DeviceTrace(w.trace))
        r = h.plan(gpu_bytes, host_bytes, w.bw_out_Bpus, w.bw_in_Bpus)
        h.prefetch()
        y = h.replay(eager=True)
        out.append((w.trace.name, h.peak, int(r.pressure_after.max()), len(r.records), int(sum(y.bytes)), y.iter_ns, y.stall_ns))
        h.close()
    return out


def main():
    import torch
    text = torch.arange(257, device="cuda").remainder(29).repeat(8, 1)               # something to learn: 0 1 2 ... 28 0 1 ...
    text = (text + torch.arange(8, device="cuda")[:, None] * 3) % 29
    model = Decoder()
    for i in range(12):
        loss, norm = model.step(text)
        if i % 3 == 0 or i == 11:
            print(f"step {i}: loss {float(loss):.2e}, gradient norm {float(norm):.2e}")
    got = model.continue_text(text[:, :40], 20)
    print("continues", int((got[:, 40:] == text[:, 40:60]).sum()), "of", got[:, 40:].numel(), "tokens as it learnt them")
    model.close()
    print("on 288 GB:")
    for name, peak, left, n, moved, it, stall in compare_plans():
        print(f"  {name}: {peak / 2**30:.0f} GiB at its peak, {left / 2**30:.0f} after {n} migrations of {moved / 2**30:.0f} GiB; "
              f"a step of {it / 1e9:.2f} s, {stall / 1e9:.2f} s of it waiting")


if __name__ == "__main__":
    main()
