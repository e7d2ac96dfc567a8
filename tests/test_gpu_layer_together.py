"""The operators around attention as a layer uses them: one behind the other, in graphs, on streams of their own, in the small decoder."""
import math

import pytest
import torch

import layercheck as L

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.fixture(scope="module")
def ops():
    from paper_2310_09443_amd import ops
    return ops


def weights(vocab, dim, inner, seed=0):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s, std: (torch.randn(*s, generator=g) * std).to(BF).cuda()                             # noqa: E731
    return dict(embed=r(vocab, dim, std=0.5), n1=(1 + r(dim, std=0.2)), b1=r(dim, std=0.2), gate=r(dim, inner, std=dim ** -0.5), up=r(dim, inner, std=dim ** -0.5),
                down=r(inner, dim, std=inner ** -0.5), n2=(1 + r(dim, std=0.2)), head=r(dim, vocab, std=dim ** -0.5))


def net(ops, w, ids, targets):
    x = ops.embed(ids, w["embed"], 2.0)
    x = x + ops.gated(ops.norm(x, w["n1"], w["b1"], center=True), w["gate"], w["up"]) @ w["down"]
    logp, ent = ops.log_probs(ops.norm(x, w["n2"]) @ w["head"], targets, entropy=True)
    return logp, ent


def net64(w, ids, targets):
    F = torch.nn.functional
    x = w["embed"][ids] * 2.0
    n = F.layer_norm(x, x.shape[-1:], w["n1"], w["b1"], 1e-6)
    x = x + (F.silu(n @ w["gate"]) * (n @ w["up"])) @ w["down"]
    lp = torch.log_softmax((x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * w["n2"]) @ w["head"], -1)
    return torch.where(targets == -100, 0.0, lp.gather(-1, targets.clamp(min=0)[..., None])[..., 0]), -(lp.exp() * lp).sum(-1)


@pytest.mark.parametrize("batch, seq", [(1, 1), (3, 37), (2, 300)])
def test_a_step(ops, batch, seq):
    """Loss and gradients of a small model.  From ids to loss and back lie 16 values rounded to bf16 one behind the other (embedding, two norms, gated, down,
    sum, head, and their gradients with dg and du); each adds at most u to the relative error in the norm, and what is in the logits counts twice: once in
    the probabilities' gradient.  24 u."""
    w = weights(97, 128, 192)
    g = torch.Generator().manual_seed(seq)
    ids, targets = torch.randint(0, 97, (batch, seq), generator=g).cuda(), torch.randint(0, 97, (batch, seq), generator=g).cuda()
    if seq > 1:
        targets[0, : seq // 2] = -100                                                                 # a padded batch
    leaves = {n: t.detach().clone().requires_grad_() for n, t in w.items()}
    logp, ent = net(ops, leaves, ids, targets)
    (logp.sum() - 0.1 * ent.sum()).backward()
    w64 = {n: L.d(t).requires_grad_() for n, t in w.items()}
    logp64, ent64 = net64(w64, ids.cpu(), targets.cpu())
    (logp64.sum() - 0.1 * ent64.sum()).backward()
    limit = 24 * L.u(BF)
    assert float((L.d(logp) - logp64.detach()).norm()) <= limit * float(logp64.detach().norm()) and float((L.d(ent) - ent64.detach()).norm()) <= limit * float(ent64.detach().norm())
    for n, t in leaves.items():
        want = w64[n].grad
        assert float((L.d(t.grad) - want).norm()) <= limit * float(want.norm()), n


def calls(ops, w, ids, targets):
    """Every forward and backward call, and what comes out."""
    x = ops.g10_embed(ids, w["embed"])
    n = ops.g10_norm(x, w["n1"], w["b1"], center=True)
    h = ops.g10_gated(n, w["gate"], w["up"])
    z = (h @ w["down"]) @ w["head"]
    logp, lse, ent, top_logp, top_ids = ops.g10_log_probs(z, targets, entropy=True, top=7)
    dz = ops.g10_log_probs_backward(logp, z, targets, lse, ent, ent)
    dh = (dz @ w["head"].t()) @ w["down"].t()
    dn, dgate, dup = ops.g10_gated_backward(dh, n, w["gate"], w["up"])
    dx, dw, db = ops.g10_norm_backward(dn, x, w["n1"], w["b1"], center=True)
    return [x, n, h, logp, lse, ent, top_logp, top_ids, dz, dn, dgate, dup, dx, dw, db, ops.g10_embed_backward(dx, ids, w["embed"].shape[0])]


def inputs(rows, seed, vocab=1000):
    g = torch.Generator().manual_seed(seed)
    return torch.randint(0, vocab, (rows,), generator=g).cuda(), torch.randint(0, vocab, (rows,), generator=g).cuda()


def test_captured_and_replayed(ops):
    """Two graphs of one pool, replayed in turn with other ids and eager work between."""
    w = weights(1000, 264, 520)
    rows = (150, 20)
    eager = {(r, s): [t.clone() for t in calls(ops, w, *inputs(r, s))] for r in rows for s in (1, 2, 3)}
    static = {r: [t.clone() for t in inputs(r, 1)] for r in rows}
    graphs, outs, pool = {}, {}, None
    for r in rows:
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            calls(ops, w, *static[r])
        torch.cuda.current_stream().wait_stream(s)
        graphs[r] = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graphs[r], pool=pool):
            outs[r] = calls(ops, w, *static[r])
        pool = pool or graphs[r].pool()
    for seed in (2, 3, 1, 2, 3):
        for r in rows:
            for t, new in zip(static[r], inputs(r, seed)):
                t.copy_(new)
            graphs[r].replay()
            for got, want in zip(outs[r], eager[r, seed]):
                assert torch.equal(got, want)
            calls(ops, w, *inputs(40, seed + 10))
            torch.cuda.synchronize()


def test_streams(ops):
    """Calls on two streams at once, with a workspace each."""
    w = weights(1000, 264, 520)
    want = [[t.clone() for t in calls(ops, w, *inputs(300, s))] for s in (1, 2)]
    ins = [inputs(300, s) for s in (1, 2)]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], [None, None]
    for _ in range(3):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i] = calls(ops, w, *ins[i])
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        for x, y in zip(a, b):
            assert torch.equal(x, y)


def test_the_same_input_twice(ops):
    """One tensor as both weights, as a table and as what is looked up in it, as gradient and input."""
    w = weights(64, 64, 64)["gate"]
    x = w[:10].contiguous()
    L.assert_gated(dict(h=ops.g10_gated(x, w, w)), L.gated(x, w, w, "silu"), BF)
    v = w.detach().clone().requires_grad_()
    ops.gated(x, v, v).sum().backward()
    one = [L.d(y) for y in ops.g10_gated_backward(torch.ones(10, 64, dtype=BF, device="cuda"), x, w, w)[1:]]
    L.assert_near(v.grad, one[0] + one[1], L.rounding(one[0] + one[1], BF))
    dx, _, _ = ops.g10_norm_backward(x, x)
    L.assert_near(dx, *L.norm(x, None, None, 1e-6, False, BF, x)["dx"])
    ids = torch.tensor([3, 3, 3], device="cuda")
    L.assert_near(ops.g10_embed_backward(x[:3], ids, 64), *L.embed_backward(x[:3], ids, 64, 1.0))


def test_rows_behind_the_last_are_left_as_they_were(ops):
    """The C ABI with outputs in a larger tensor: nothing is written outside the outputs' elements."""
    import ctypes as C
    lib, guard, stream = ops._load(), 7.0, torch.cuda.current_stream().cuda_stream
    rows, dim, inner = 37, 72, 136
    big = lambda r, c, t=BF: torch.full((r + 20, c + 24), guard, dtype=t, device="cuda")                # noqa: E731
    x, wg, wu = (torch.randn(a, b, device="cuda").to(BF) for a, b in ((rows, dim), (dim, inner), (dim, inner)))

    def kept(t, r, c):
        t = t.clone()
        t[:r, :c] = guard
        return bool((t == guard).all())
    h, dx, dg, du, y, e, dt, dl = big(rows, inner), big(rows, dim), big(dim, inner), big(dim, inner), big(rows, dim), big(rows, dim), big(50, dim), big(rows, dim)
    dh = torch.randn(rows, inner, device="cuda").to(BF)
    p = lambda t: t.data_ptr()                                                                          # noqa: E731
    room = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    a = ops._Gated(x=p(x), gate=p(wg), up=p(wu), h=p(h), dh=p(dh), dx=p(dx), dgate=p(dg), dup=p(du), x_stride=dim, gate_stride=inner, up_stride=inner, h_stride=h.stride(0), dh_stride=inner,
                   dx_stride=dx.stride(0), dw_stride=dg.stride(0), tokens=rows, dim=dim, inner=inner, act=0, type=ops.BF16)
    assert lib.g10_gated(C.byref(a), p(room), room.numel(), stream) == 0 and lib.g10_gated_backward(C.byref(a), p(room), room.numel(), stream) == 0
    assert torch.equal(h[:rows, :inner], ops.g10_gated(x, wg, wu))
    for got, want in zip((dx[:rows, :dim], dg[:dim, :inner], du[:dim, :inner]), ops.g10_gated_backward(dh, x, wg, wu)):
        assert torch.equal(got, want)
    n = ops._Norm(x=p(x), out=p(y), x_stride=dim, out_stride=y.stride(0), rows=rows, dim=dim, eps=1e-6, type=ops.BF16, weight_type=ops.BF16)
    assert lib.g10_norm(C.byref(n), stream) == 0 and torch.equal(y[:rows, :dim], ops.g10_norm(x))
    ids = torch.randint(0, 50, (rows,), device="cuda")
    m = ops._Embed(ids=p(ids), table=p(wg), out=p(e), dout=p(x), dtable=p(dt), table_stride=inner, out_stride=e.stride(0), dout_stride=dim, dtable_stride=dt.stride(0),
                   tokens=rows, vocab=50, dim=dim, scale=1.0, type=ops.BF16, ids_64=1)
    assert lib.g10_embed(C.byref(m), stream) == 0 and lib.g10_embed_backward(C.byref(m), p(room), room.numel(), stream) == 0
    assert torch.equal(e[:rows, :dim], wg[:50, :dim][ids]) and torch.equal(dt[:50, :dim], ops.g10_embed_backward(x, ids, 50))
    lse, dlogp = torch.empty(rows, device="cuda"), torch.randn(rows, device="cuda")
    q = ops._LogProbs(logits=p(x), tokens=p(ids), logp=p(torch.empty_like(lse)), lse=p(lse), dlogp=p(dlogp), dlogits=p(dl), logits_stride=dim, dlogits_stride=dl.stride(0),
                      rows=rows, vocab=dim, scale=1.0, ignore=-100, type=ops.BF16)
    assert lib.g10_log_probs(C.byref(q), None, 0, stream) == 0 and lib.g10_log_probs_backward(C.byref(q), stream) == 0
    assert torch.equal(dl[:rows, :dim], ops.g10_log_probs_backward(dlogp, x, ids, lse))
    torch.cuda.synchronize()
    assert kept(h, rows, inner) and kept(dx, rows, dim) and kept(dg, dim, inner) and kept(du, dim, inner) and kept(y, rows, dim) and kept(e, rows, dim)
    assert kept(dt, 50, dim) and kept(dl, rows, dim)


def test_in_place(ops):
    """What the header allows to be written over its input."""
    import ctypes as C
    lib, stream = ops._load(), torch.cuda.current_stream().cuda_stream
    for dim in (72, 1100):
        x, dy = (torch.randn(50, dim, device="cuda").to(BF) for _ in range(2))
        t = torch.randint(0, dim, (50,), device="cuda")
        want = ops.g10_norm(x, center=True), ops.g10_norm_backward(dy, x, center=True)[0]
        _, lse, _, _, _ = ops.g10_log_probs(x, t)
        grad = ops.g10_log_probs_backward(lse, x, t, lse)
        y, g, z = x.clone(), dy.clone(), x.clone()
        n = ops._Norm(x=y.data_ptr(), out=y.data_ptr(), x_stride=dim, out_stride=dim, rows=50, dim=dim, eps=1e-6, center=1, type=ops.BF16, weight_type=ops.BF16)
        assert lib.g10_norm(C.byref(n), stream) == 0 and torch.equal(y, want[0])
        n.x, n.dy, n.out, n.dy_stride = x.data_ptr(), g.data_ptr(), g.data_ptr(), dim
        assert lib.g10_norm_backward(C.byref(n), None, 0, stream) == 0 and torch.equal(g, want[1])
        q = ops._LogProbs(logits=z.data_ptr(), tokens=t.data_ptr(), lse=lse.data_ptr(), dlogp=lse.data_ptr(), dlogits=z.data_ptr(), logits_stride=dim, dlogits_stride=dim,
                          rows=50, vocab=dim, scale=1.0, ignore=-100, type=ops.BF16)
        assert lib.g10_log_probs_backward(C.byref(q), stream) == 0 and torch.equal(z, grad)


def test_long_rows_of_memory(ops):
    """Places past 2^31 elements: the last rows of a tensor of 4.5 GB."""
    rows, dim = 34000, 66000
    x = torch.zeros(rows, dim, dtype=BF, device="cuda")
    x[-3:] = torch.randn(3, dim, device="cuda").to(BF)
    t = torch.full((rows,), 5, device="cuda")
    logp, lse, _, _, ids = ops.g10_log_probs(x, t, top=3)
    want, wids = L.log_probs(x[-3:], t[-3:], 1.0, -100, 3)
    L.assert_near(lse[-3:], *want["lse"])
    L.assert_near(logp[-3:], *want["logp"])
    assert torch.equal(ids[-3:].cpu(), wids) and abs(float(lse[0]) - math.log(dim)) < 1e-5
    d = ops.g10_log_probs_backward(logp, x, t, lse)
    L.assert_near(d[-3:], *L.log_probs(x[-3:], t[-3:], 1.0, -100, 0, logp[-3:])[0]["dlogits"])
    del d
    v = x.view(-1)[: (1 << 31) + 4096 * 25].view(-1, 4096)                                              # 524313 rows of 4096
    ids = torch.tensor([0, v.shape[0] - 1, v.shape[0] - 2], device="cuda")
    L.assert_near(ops.g10_embed(ids, v), L.d(v[ids]), torch.zeros(3, 4096, dtype=torch.float64))
    n = ops.g10_norm(v)
    L.assert_near(n[-2:], *L.norm(v[-2:], None, None, 1e-6, False, BF)["y"])


def test_the_small_decoder_goes_through_them(ops):
    """A step gives every weight a gradient, and a reply is made of the likeliest tokens."""
    from paper_2310_09443_amd import lean
    m = lean.Decoder(vocab=50, dim=64, layers=1, heads=2, kv_heads=1, inner=96, max_len=64)
    ids = torch.randint(0, 50, (2, 20), device="cuda")
    loss, norm = m.step(ids)
    assert bool(torch.isfinite(loss)) and float(norm) > 0
    assert all(t.grad is not None and bool(torch.isfinite(t.grad).all()) for w in m.layers for t in w.values())
    with torch.no_grad():
        new = m.continue_text(ids, 3)[:, 20:]
        z = m.logits(torch.cat([ids, new], 1)).float()[:, 19:22]
    assert ((z.amax(-1) - z.gather(2, new[..., None])[..., 0]) <= 0.05 * z.abs().amax(-1)).all()          # (what bf16 loses between one pass and three)
    m.close()
