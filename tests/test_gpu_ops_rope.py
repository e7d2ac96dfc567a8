"""Norms of queries and keys with the rotation, against the 64-bit formulas: every rotation, type, layout and size it can go wrong at."""
import pytest
import torch

import opscheck as O

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    from paper_2310_09443_amd import ops
    return ops


def make(batch, seq, hq, hk, dim, rot, dtype, weights=True, wtype=None, seed=0, sliced=False, n_pos=64):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)                                          # noqa: E731
    if sliced:
        x = (r(batch, seq, hq + 2 * hk, dim) * 2).to(dtype).cuda()
        q, k = x[:, :, :hq], x[:, :, hq:hq + hk]
    else:
        q, k = (r(batch, seq, hq, dim) * 2).to(dtype).cuda(), (r(batch, seq, hk, dim) * 0.01).to(dtype).cuda()
    qw, kw = ((1 + 0.3 * r(dim)).to(wtype or dtype).cuda() for _ in range(2)) if weights else (None, None)
    table = torch.rand(n_pos, rot, generator=g).mul(2).sub(1).cuda()
    pos = torch.randint(0, n_pos, (batch, seq), generator=g, dtype=torch.int32).cuda()
    dq, dk = (torch.randn(t.shape, generator=g).to(dtype).cuda() for t in (q, k))
    return dict(q=q, k=k, table=table, positions=pos, q_weight=qw, k_weight=kw), (dq, dk)


def check(ops, a, grads, eps=1e-6, interleaved=False):
    dtype = a["q"].dtype
    got = ops.g10_norm_rope(**a, eps=eps, interleaved=interleaved)
    back = ops.g10_norm_rope_backward(*grads, **a, eps=eps, interleaved=interleaved)
    for i, n in enumerate(("q", "k")):
        w = a[n + "_weight"]
        want, tol = O.rope(a[n], w, a["table"], a["positions"], eps, interleaved, dtype)
        O.assert_near(got[i], want, tol, n)
        dx, tx, dw, tw = O.rope_backward(grads[i], a[n], w, a["table"], a["positions"], eps, interleaved, dtype)
        O.assert_near(back[i], dx, tx, "d" + n)
        if w is not None:
            O.assert_near(back[2 + i], dw, tw + O.rounding(dw, w.dtype), "dw" + n)
        else:
            assert back[2 + i] is None


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim, rot", [(64, 64), (128, 128), (256, 256), (128, 32), (80, 48), (8, 0), (40, 40), (192, 64), (24, 16),
                                      (7, 6), (1, 0), (250, 250), (72, 50), (129, 2)])
def test_dims(ops, dim, rot, interleaved, dtype):
    check(ops, *make(2, 5, 3, 2, dim, rot, dtype, seed=dim + rot), interleaved=interleaved)


@pytest.mark.parametrize("batch, seq, hq, hk", [(1, 1, 1, 1), (1, 1, 32, 8), (3, 1, 5, 5), (1, 77, 9, 3), (2, 130, 16, 1), (1, 700, 24, 8)])
def test_sizes(ops, batch, seq, hq, hk):
    check(ops, *make(batch, seq, hq, hk, 64, 64, torch.bfloat16, seed=seq))


def test_many_rows(ops):
    """More rows than a backward pass has groups, and the task of eight heads: 2049 tokens of 19 heads."""
    check(ops, *make(1, 2049, 13, 6, 128, 128, torch.bfloat16, seed=9))
    check(ops, *make(1, 6001, 5, 3, 12, 12, torch.float32, seed=10))


@pytest.mark.parametrize("dim", [64, 20])
def test_layouts(ops, dim):
    check(ops, *make(2, 9, 4, 2, dim, dim // 4 * 2, torch.float16, sliced=True))            # slices of one projection
    check(ops, *make(2, 9, 4, 2, dim, dim // 4 * 2, torch.bfloat16, weights=False))
    check(ops, *make(2, 9, 4, 2, dim, dim // 4 * 2, torch.bfloat16, wtype=torch.float32))
    a, gr = make(2, 9, 4, 2, dim, dim // 4 * 2, torch.bfloat16)
    a["positions"] = a["positions"].long()
    check(ops, a, gr)
    a["q"] = torch.stack([a["q"], a["q"]], -1)[..., 0]                                       # last dimension not contiguous
    a["k"] = torch.cat([a["k"].reshape(-1)[:1], a["k"].reshape(-1)])[1:].view(a["k"].shape)  # not aligned
    check(ops, a, (gr[0].transpose(0, 1).contiguous().transpose(0, 1), gr[1].expand(gr[1].shape)))
    t = {n: (x[0] if n in ("q", "k", "positions") else x) for n, x in a.items()}              # [token, head, dim]
    check(ops, t, (gr[0][0], gr[1][0]))


def test_one_of_both_and_none(ops):
    a, gr = make(1, 6, 4, 2, 64, 64, torch.bfloat16)
    both = ops.g10_norm_rope(**a)
    q, none = ops.g10_norm_rope(a["q"], None, a["table"], a["positions"], a["q_weight"])
    assert none is None and torch.equal(q, both[0])
    none, k = ops.g10_norm_rope(None, a["k"], a["table"], a["positions"], None, a["k_weight"])
    assert none is None and torch.equal(k, both[1])
    e = {n: (x[:, :0] if n in ("q", "k", "positions") else x) for n, x in a.items()}          # no tokens
    got = ops.g10_norm_rope(**e)
    back = ops.g10_norm_rope_backward(gr[0][:, :0], gr[1][:, :0], **e)
    assert got[0].shape[1] == 0 and not back[2].any() and not back[3].any()


def test_positions_outside_the_table_are_seen(ops):
    a, gr = make(1, 5, 3, 2, 128, 64, torch.bfloat16)
    for dim64 in (False, True):
        p = a["positions"].clone().long() if dim64 else a["positions"].clone()
        p[0, 1], p[0, 3] = -1, 64
        if dim64:
            p[0, 3] = 1 << 40
        got = ops.g10_norm_rope(**dict(a, positions=p))
        back = ops.g10_norm_rope_backward(*gr, **dict(a, positions=p))
        for x in (*got, *back[:2]):
            assert torch.isnan(x[0, [1, 3]]).all() and not torch.isnan(x[0, [0, 2, 4]]).any()
        assert torch.isnan(back[2]).any()


def test_zero_rows_and_large_values(ops):
    a, gr = make(1, 4, 2, 2, 64, 64, torch.float32)
    a["q"][0, 1] = 0
    a["k"][0, 2] = 1e15
    check(ops, a, gr)


def test_gradients_by_autograd_and_differences(ops):
    a, (dq, dk) = make(1, 7, 3, 1, 32, 32, torch.float32, seed=3)
    leaves = {n: a[n].clone().requires_grad_() for n in ("q", "k", "q_weight", "k_weight")}
    q, k = ops.norm_rope(**dict(a, **leaves), eps=1e-3)
    torch.autograd.backward((q, k), (dq, dk))
    want = ops.g10_norm_rope_backward(dq, dk, **a, eps=1e-3)
    for n, w in zip(leaves, want):
        assert torch.equal(leaves[n].grad, w), n
    loss = lambda b: sum(float((x.double() * y.double()).sum()) for x, y in zip(ops.g10_norm_rope(**b, eps=1e-3), (dq, dk)))    # noqa: E731
    for n in leaves:
        # k's values are of the size 0.01, the square of eps' root beside it: steps of a hundredth of a value
        way, h = torch.randn(a[n].shape, generator=torch.Generator().manual_seed(1)).cuda(), 0.01 * float(a[n].abs().mean())
        slope = (loss(dict(a, **{n: a[n] + h * way})) - loss(dict(a, **{n: a[n] - h * way}))) / (2 * h)
        size = float((leaves[n].grad.double().abs() * way.double().abs()).sum())
        # third-order term of the difference: (h way / value)^2 of the magnitudes; roundings: 2^-20 of the loss' terms over h
        noise = 2.0 ** -20 * float(dq.abs().sum() + dk.abs().sum()) * 3 / h
        assert abs(slope - float((leaves[n].grad.double() * way.double()).sum())) < 5e-3 * size + noise, n


def test_refusals(ops):
    a, gr = make(1, 3, 2, 2, 64, 64, torch.bfloat16)
    for bad in (dict(q=a["q"].float()), dict(k=a["k"][:, :2]), dict(table=a["table"].double()), dict(table=a["table"][:, :63]),
                dict(table=torch.zeros(4, 66, device="cuda")), dict(positions=a["positions"].float()), dict(positions=a["positions"][:, :2]),
                dict(q_weight=a["q_weight"][:8]), dict(q_weight=a["q_weight"].float()), dict(eps=-1), dict(table=a["table"][:0]),
                dict(q=a["q"].double(), k=a["k"].double()), dict(positions=a["positions"].cpu())):
        with pytest.raises(ValueError):
            ops.g10_norm_rope(**dict(a, **bad))
    with pytest.raises(ValueError):
        ops.g10_norm_rope_backward(gr[0], gr[0][:, :1], **a)


def test_same_every_time_other_streams_and_graphs(ops):
    a, gr = make(2, 300, 8, 2, 128, 128, torch.bfloat16, seed=5)
    first = (*ops.g10_norm_rope(**a), *ops.g10_norm_rope_backward(*gr, **a))
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        again = (*ops.g10_norm_rope(**a), *ops.g10_norm_rope_backward(*gr, **a))
    s.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(first, again))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        inside = (*ops.g10_norm_rope(**a), *ops.g10_norm_rope_backward(*gr, **a))
    for k in range(4):
        a["q"].mul_(1.5)
        gr[1].add_(0.25)
        g.replay()
        eager = (*ops.g10_norm_rope(**a), *ops.g10_norm_rope_backward(*gr, **a))
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(inside, eager)), k
