"""Attention against the 64-bit formulas: lengths from none to several tiles, windows, sinks, groups of heads, packed and padded
sequences, rows that see nothing, and what lies behind a sequence's end."""
import pytest
import torch

import opscheck as O

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    from paper_2310_09443_amd import ops
    return ops


def make(lead_q, lead_k, heads, kv, dim, dtype, seed=0, do_scale=1.0):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)                                          # noqa: E731
    q, k, v = (r(*lead_q, heads, dim) * 1.5).to(dtype), r(*lead_k, kv, dim).to(dtype), r(*lead_k, kv, dim).to(dtype)
    return [t.cuda() for t in (q, k, v, (r(*lead_q, heads, dim) * do_scale).to(dtype))]


def check(ops, q, k, v, do=None, causal=True, window=0, sinks=0, scale=None, **where):
    args = dict(causal=causal, window=window, sinks=sinks, scale=scale, **where)
    cpu = {n: (t.cpu() if isinstance(t, torch.Tensor) else t) for n, t in where.items() if n not in ("max_q", "max_k")}
    want = O.attention(q.cpu(), k.cpu(), v.cpu(), do.cpu() if do is not None else None, causal, window, sinks, scale, **cpu)
    o, lse = ops.g10_attention(q, k, v, **args)
    got = dict(o=o, lse=lse)
    if do is not None:
        got.update(zip(("dq", "dk", "dv"), ops.g10_attention_backward(do, q, k, v, o, lse, **args)))
    for n, x in got.items():
        O.assert_near(x, *want[n], n)
    return got


MASKS = [(True, 0, 0), (True, 1, 0), (True, 37, 0), (True, 70, 5), (True, 3, 100), (False, 0, 0), (False, 40, 3), (False, 1, 0)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("causal, window, sinks", MASKS)
@pytest.mark.parametrize("nq, nk", [(1, 1), (33, 33), (64, 64), (129, 129), (200, 333), (257, 70)])
def test_lengths_and_masks(ops, nq, nk, causal, window, sinks, dtype):
    check(ops, *make((2, nq), (2, nk), 2, 1, 64, dtype, seed=nq + nk), causal=causal, window=window, sinks=sinks)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dim", [8, 24, 40, 64, 72, 96, 128])
def test_dims(ops, dim, dtype):
    check(ops, *make((1, 150), (1, 150), 2, 2, dim, dtype, seed=dim))
    check(ops, *make((1, 100), (1, 181), 3, 1, dim, dtype, seed=dim), causal=False, window=90, sinks=70)


@pytest.mark.parametrize("heads, kv", [(1, 1), (8, 1), (6, 3), (16, 16), (9, 9), (40, 8)])
def test_groups_of_heads(ops, heads, kv):
    check(ops, *make((3, 70), (3, 70), heads, kv, 64, torch.bfloat16, seed=heads))
    check(ops, *make((3, 3), (3, 140), heads, kv, 128, torch.bfloat16, seed=heads))


@pytest.mark.parametrize("nq", [1, 2, 5])
@pytest.mark.parametrize("nk", [1, 16, 127, 128, 500, 1500])
@pytest.mark.parametrize("window, sinks", [(0, 0), (100, 4), (1, 0)])
def test_new_tokens_on_a_cache(ops, nq, nk, window, sinks):
    q, k, v, _ = make((4, nq), (4, nk), 8, 2, 128, torch.bfloat16, seed=nk + nq)
    k_len = torch.tensor([nk, 0, max(1, nk // 3), max(1, nk - 1)], dtype=torch.int32).cuda()
    for b, n in enumerate(k_len.tolist()):                            # what lies behind a sequence's end is not read
        k[b, n:] = float("nan")
        v[b, n:] = float("inf")
    check(ops, q, k, v, window=window, sinks=sinks, k_len=k_len)


def test_keys_behind_the_end_get_zeros(ops):
    q, k, v, do = make((3, 90), (3, 200), 4, 2, 64, torch.float16, seed=4)
    k_len = torch.tensor([200, 0, 65], dtype=torch.int32).cuda()
    k[2, 65:] = float("inf")
    v[2, 65:] = float("nan")
    got = check(ops, q, k, v, do, k_len=k_len)
    assert not got["dk"][2, 65:].any() and not got["dv"][1].any() and not got["dq"][1].any() and not got["o"][1].any()
    assert (got["lse"][1] == -float("inf")).all()


@pytest.mark.parametrize("dim, dtype", [(64, torch.float16), (128, torch.bfloat16), (80, torch.bfloat16)])
@pytest.mark.parametrize("causal, window, sinks", [(True, 0, 0), (True, 50, 4), (False, 0, 0)])
def test_packed(ops, dim, dtype, causal, window, sinks):
    n = [130, 1, 0, 64, 257, 31]
    at = torch.tensor([0] + n).cumsum(0).to(torch.int32).cuda()
    total = int(at[-1])
    q, k, v, do = make((total,), (total,), 4, 2, dim, dtype, seed=dim)
    args = dict(causal=causal, window=window, sinks=sinks, q_start=at, k_start=at)
    first = check(ops, q, k, v, do, **args, max_q=257, max_k=257)
    # lengths that are told wrong, or not at all, cut the work differently: the same values
    for most in (1, 130, None):
        o, lse = ops.g10_attention(q, k, v, **args, max_q=most, max_k=most)
        got = dict(zip(("o", "lse", "dq", "dk", "dv"), (o, lse, *ops.g10_attention_backward(do, q, k, v, o, lse, **args, max_q=most, max_k=most))))
        for name, x in got.items():
            assert torch.equal(x, first[name]), (most, name)


def test_packed_queries_and_keys_of_other_lengths(ops):
    nq, nk = [3, 0, 40, 1], [200, 17, 20, 0]
    a, b = (torch.tensor([0] + n).cumsum(0).to(torch.int32).cuda() for n in (nq, nk))
    q, k, v, do = make((int(a[-1]),), (int(b[-1]),), 6, 2, 64, torch.bfloat16)
    check(ops, q, k, v, do, q_start=a, k_start=b, max_q=40, max_k=200)
    check(ops, q, k, v, do, q_start=a, k_start=b, max_q=40, max_k=200, window=9, sinks=2)


def test_starts_outside_the_tensors_stay_inside(ops):
    """Numbers that point outside are moved to the border: what such a sequence holds is cut, nothing else is touched."""
    q, k, v, do = make((100,), (100,), 2, 2, 64, torch.bfloat16)
    bad = torch.tensor([-5, 60, 1 << 30, 40], dtype=torch.int32).cuda()
    good = torch.tensor([0, 60, 100, 100], dtype=torch.int32).cuda()
    for x, y in zip(ops.g10_attention(q, k, v, q_start=bad, k_start=bad, max_q=100, max_k=100),
                    ops.g10_attention(q, k, v, q_start=good, k_start=good, max_q=100, max_k=100)):
        assert torch.equal(x, y)
    q, k, v, do = make((2, 30), (2, 50), 2, 2, 64, torch.bfloat16)
    x = ops.g10_attention(q, k, v, k_len=torch.tensor([-3, 1 << 30], dtype=torch.int32).cuda())[0]
    y = ops.g10_attention(q, k, v, k_len=torch.tensor([0, 50], dtype=torch.int32).cuda())[0]
    assert torch.equal(x, y)


def test_layouts(ops):
    g = torch.Generator().manual_seed(2)
    qkv = torch.randn(2, 75, 8, 64, generator=g).to(torch.bfloat16).cuda()            # slices of one projection
    do = torch.randn(2, 75, 4, 64, generator=g).to(torch.bfloat16).cuda()
    q, k, v = qkv[:, :, :4], qkv[:, :, 4:6], qkv[:, :, 6:]
    want = check(ops, q, k, v, do)
    by_head = [t.transpose(1, 2).contiguous().transpose(1, 2) for t in (q, k, v, do)]   # heads before tokens
    odd = [torch.cat([t.reshape(-1)[:1], t.reshape(-1)])[1:].view(t.shape) for t in (q, k, v, do)]   # not aligned
    last = [torch.stack([t, t], -1)[..., 0] for t in (q, k, v, do)]                      # last dimension not contiguous
    for a in (by_head, odd, last):
        o, lse = ops.g10_attention(*a[:3])
        got = dict(zip(("o", "lse", "dq", "dk", "dv"), (o, lse, *ops.g10_attention_backward(a[3], *a[:3], o, lse))))
        for n, x in got.items():
            assert torch.equal(x, want[n]), n
    one = check(ops, q, k[:, :, :1].expand(2, 75, 1, 64), v[:, :, :1], do)
    flipped = ops.g10_attention(q.flip(1), k[:, :, :1], v[:, :, :1], causal=False)[0].flip(1)
    assert torch.equal(flipped, ops.g10_attention(q, k[:, :, :1], v[:, :, :1], causal=False)[0]) and one["o"].shape == q.shape


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_scores_of_all_sizes(ops, dtype):
    """Scores that leave one key, scores that are all alike, a scale of one's own, gradients as small as they get."""
    q, k, v, do = make((1, 160), (1, 160), 2, 1, 64, dtype, seed=8)
    check(ops, q * 8, k * 4, v, do)
    check(ops, q * 0, k, v, do)
    check(ops, q, k, v, do, scale=0.01)
    check(ops, q, k, v, do * 2.0 ** -12, scale=1.0)
    check(ops, q, k, v * 16, do * 0, causal=False)


def test_a_late_key_that_outweighs_all_before(ops):
    """The running maximum rises by far in the last tile, and falls never."""
    q, k, v, do = make((1, 300), (1, 300), 1, 1, 64, torch.bfloat16, seed=1)
    k[0, 290] = q[0, 295, 0] * 6
    k[0, 3] = q[0, 120, 0] * 3
    check(ops, q, k, v, do)
    check(ops, q, k, v, do, causal=False)


def test_long_offsets(ops):
    """A cache whose rows lie more than 2^32 bytes from its beginning."""
    dim, heads, seq = 128, 1, 4
    big = torch.empty((3 << 30) // 2 + (1 << 20), dtype=torch.bfloat16, device="cuda")
    row = 1 << 20                                                     # elements between tokens
    k = big.as_strided((1, 1500, heads, dim), (0, row, dim, 1))
    v = big.as_strided((1, 1500, heads, dim), (0, row, dim, 1), 4096)
    q, kk, vv, _ = make((1, seq), (1, 1500), heads, heads, dim, torch.bfloat16)
    k.copy_(kk)
    v.copy_(vv)
    got = ops.g10_attention(q, k, v)
    want = ops.g10_attention(q, kk, vv)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_gradients_by_autograd(ops):
    q, k, v, do = make((2, 90), (2, 90), 4, 2, 64, torch.float16, seed=6)
    leaves = [t.clone().requires_grad_() for t in (q, k, v)]
    o = ops.attention(*leaves, window=20, sinks=1)
    o.backward(do)
    fo, lse = ops.g10_attention(q, k, v, window=20, sinks=1)
    assert torch.equal(o, fo)
    for x, y in zip(leaves, ops.g10_attention_backward(do, q, k, v, fo, lse, window=20, sinks=1)):
        assert torch.equal(x.grad, y)
    # a gradient that is broadcast, as that of a sum is
    leaves = [t.clone().requires_grad_() for t in (q, k, v)]
    ops.attention(*leaves).sum().backward()
    fo, lse = ops.g10_attention(q, k, v)
    for x, y in zip(leaves, ops.g10_attention_backward(torch.ones_like(do), q, k, v, fo, lse)):
        assert torch.equal(x.grad, y)


def test_empty(ops):
    q, k, v, do = make((2, 0), (2, 5), 2, 2, 64, torch.bfloat16)
    o, lse = ops.g10_attention(q, k, v)
    assert o.shape == q.shape and not any(x.any() for x in ops.g10_attention_backward(do, q, k, v, o, lse))
    q, k, v, do = make((2, 5), (2, 0), 2, 2, 64, torch.bfloat16)
    o, lse = ops.g10_attention(q, k, v)
    assert not o.any() and (lse == -float("inf")).all()
    assert not any(x.any() for x in ops.g10_attention_backward(do, q, k, v, o, lse))
    q, k, v, do = make((0, 5), (0, 5), 2, 2, 64, torch.bfloat16)
    assert ops.g10_attention(q, k, v)[0].shape == q.shape


def test_refusals(ops):
    q, k, v, do = make((1, 8), (1, 8), 4, 2, 64, torch.bfloat16)
    at = torch.tensor([0, 8], dtype=torch.int32).cuda()
    for bad in (dict(q=q.float()), dict(k=k.half()), dict(v=v[:, :4]), dict(q=q[..., :60], k=k[..., :60], v=v[..., :60]), dict(k=k[:, :, :0], v=v[:, :, :0]),
                dict(q=q[:, :, :3]), dict(scale=-1.0), dict(scale=0.0), dict(window=-1), dict(sinks=-1), dict(q_start=at), dict(q_start=at, k_start=at),
                dict(k_len=at), dict(k_len=at[:1].long()), dict(q=q[0], k=k[0], v=v[0]), dict(q=q[0], k=k[0], v=v[0], q_start=at, k_start=at[:1])):
        with pytest.raises(ValueError):
            ops.g10_attention(**dict(dict(q=q, k=k, v=v), **bad))
    o, lse = ops.g10_attention(q, k, v)
    for bad in (dict(do=do[:, :3]), dict(o=o.float()), dict(lse=lse[:, :2]), dict(lse=lse.double())):
        with pytest.raises(ValueError):
            ops.g10_attention_backward(**dict(dict(do=do, q=q, k=k, v=v, o=o, lse=lse), **bad))


def test_same_every_time_other_streams_and_graphs(ops):
    q, k, v, do = make((2, 400), (2, 400), 8, 2, 128, torch.bfloat16, seed=5)
    tok, cache_k, cache_v, _ = make((2, 1), (2, 3000), 8, 2, 128, torch.float16, seed=6)

    def work():
        o, lse = ops.g10_attention(q, k, v, window=100, sinks=3)
        return (o, lse, *ops.g10_attention_backward(do, q, k, v, o, lse, window=100, sinks=3), *ops.g10_attention(tok, cache_k, cache_v),
                *ops.g10_attention_backward(tok, tok, cache_k, cache_v, *ops.g10_attention(tok, cache_k, cache_v)))

    first = work()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        again = work()
    s.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(first, again))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        inside = work()
    for n in range(4):
        q.mul_(0.9)
        v.add_(0.125)
        cache_k.mul_(1.1)
        g.replay()
        eager = work()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(inside, eager)), n


@pytest.mark.parametrize("dim, dtype", [(64, torch.float16), (128, torch.bfloat16)])
@pytest.mark.parametrize("nq, nk, causal, window, sinks", [
    (1, 500, True, 100, 4), (1, 500, True, 100, 0), (1, 70, False, 9, 40), (40, 500, True, 30, 5), (40, 500, True, 1, 0), (40, 130, False, 20, 70),
    (130, 500, True, 64, 33), (130, 500, False, 1, 0), (300, 70, True, 0, 0), (300, 70, True, 20, 3), (300, 70, False, 33, 0), (140, 1, True, 1, 0)])
def test_what_nobody_sees_may_hold_anything(ops, dim, dtype, nq, nk, causal, window, sinks):
    """Keys between the sinks and the first window, as a cache that is written round and round leaves them, and queries before the first key."""
    q, k, v, do = make((2, nq), (2, nk), 4, 2, dim, dtype, seed=nq + nk)
    args = dict(causal=causal, window=window, sinks=sinks)
    seen = O.visible(nq, nk, causal, window, sinks)
    blind, unseen = ~seen.any(1), ~seen.any(0)
    assert blind.any() or unseen.any()

    def run(q, k, v, do):
        o, lse = ops.g10_attention(q, k, v, **args)
        return (o, lse, *ops.g10_attention_backward(do, q, k, v, o, lse, **args))

    want = run(q, k, v, do)
    for value in (float("nan"), float("inf"), -torch.finfo(dtype).max):
        for t in (k, v):
            t[:, unseen.cuda()] = value
        for t in (q, do):
            t[:, blind.cuda()] = value
        for x, y in zip(run(q, k, v, do), want):
            assert torch.equal(x, y)


@pytest.mark.parametrize("heads, kv, dim, dtype", [(8, 2, 128, torch.bfloat16), (4, 4, 64, torch.float16), (32, 1, 40, torch.bfloat16)])
@pytest.mark.parametrize("nq, nk, window, sinks", [(9, 2000, 0, 0), (17, 1100, 0, 0), (70, 3000, 0, 0), (70, 3000, 1200, 5), (130, 2500, 900, 0), (33, 2600, 40, 4)])
def test_few_queries_and_many_keys(ops, nq, nk, window, sinks, heads, kv, dim, dtype):
    """Blocks of queries and heads whose keys are cut into shares: sequences of unlike lengths, one without a key, one shorter than the queries."""
    q, k, v, _ = make((5, nq), (5, nk), heads, kv, dim, dtype, seed=nq + nk)
    k_len = torch.tensor([nk, 0, max(1, nq // 2), nk - 33, 700], dtype=torch.int32).cuda()
    for b, n in enumerate(k_len.tolist()):
        k[b, n:] = float("nan")
        v[b, n:] = float("inf")
    check(ops, q, k, v, window=window, sinks=sinks, k_len=k_len)
    check(ops, q[:1], k[:1], v[:1], window=window, sinks=sinks, causal=False)


def test_few_packed_queries_and_many_keys(ops):
    nq, nk = [20, 0, 1, 64, 3], [3000, 900, 1500, 64, 0]
    at = [torch.tensor([0] + n).cumsum(0).to(torch.int32).cuda() for n in (nq, nk)]
    q, k, v, _ = make((sum(nq),), (sum(nk),), 8, 2, 64, torch.bfloat16)
    first = check(ops, q, k, v, q_start=at[0], k_start=at[1], max_q=64, max_k=3000)
    for most in (1, 30, None):
        o, lse = ops.g10_attention(q, k, v, q_start=at[0], k_start=at[1], max_q=most, max_k=most)
        assert torch.equal(o, first["o"]) and torch.equal(lse, first["lse"])


def test_more_sequences_than_are_cut(ops):
    """300 sequences: whole blocks; 200: shares, most of them shorter than a share."""
    for n in (300, 200):
        q, k, v, _ = make((n, 1), (n, 900), 4, 1, 64, torch.bfloat16, seed=n)
        k_len = (torch.arange(n, dtype=torch.int32) * 37 % 901).cuda()
        check(ops, q, k, v, k_len=k_len)


@pytest.mark.parametrize("dim, dtype", [(64, torch.float16), (128, torch.bfloat16)])
@pytest.mark.parametrize("n, causal, window", [(7, True, 0), (60, True, 0), (380, False, 0), (512, False, 0), (760, False, 0), (1200, True, 500)])
def test_gradients_are_off_by_little_more_than_their_rounding(ops, n, causal, window, dim, dtype):
    """Their own rounding, once more as much from the 16-bit factors of their products, a quarter of it from delta: 1.5 times one rounding in all."""
    q, k, v, do = make((2, n), (2, n), 4, 2, dim, dtype, seed=n)
    want = O.attention(q.cpu(), k.cpu(), v.cpu(), do.cpu(), causal, window, 0)
    o, lse = ops.g10_attention(q, k, v, causal=causal, window=window)
    for name, x in zip(("dq", "dk", "dv"), ops.g10_attention_backward(do, q, k, v, o, lse, causal=causal, window=window)):
        exact = want[name][0]
        once = (exact.to(dtype).double() - exact).norm()
        assert (O.d(x) - exact).norm() <= 1.5 * once, name


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_gradients_of_keys_in_shares(ops, dtype):
    """Few tiles of keys with many queries each: cut into shares, wherever the cuts fall."""
    check(ops, *make((1, 1200), (1, 1200), 8, 1, 128, dtype, seed=1))
    check(ops, *make((2, 640), (2, 640), 16, 1, 64, dtype, seed=2), causal=False, window=100)
    q, k, v, do = make((3, 150), (3, 400), 12, 1, 128, dtype, seed=3)
    got = check(ops, q, k, v, do, causal=False, k_len=torch.tensor([400, 0, 129], dtype=torch.int32).cuda())
    assert not got["dk"][1].any() and not got["dv"][2, 129:].any()
    nq, nk = [0, 500, 1, 0, 300, 640], [90, 500, 700, 0, 40, 640]        # rows that see few keys, sinks that all see
    at = [torch.tensor([0] + n).cumsum(0).to(torch.int32).cuda() for n in (nq, nk)]
    args = make((sum(nq),), (sum(nk),), 16, 2, 64, dtype, seed=4)
    check(ops, *args, q_start=at[0], k_start=at[1], window=30, sinks=140)
    check(ops, *args, q_start=at[0], k_start=at[1], window=30, sinks=5, max_q=640, max_k=700)


def test_gradients_of_keys_in_shares_of_many_sequences(ops):
    n = [(i * 37) % 80 if i % 7 else 0 for i in range(600)]
    at = torch.tensor([0] + n).cumsum(0).to(torch.int32).cuda()
    check(ops, *make((sum(n),), (sum(n),), 64, 1, 72, torch.bfloat16, seed=5), q_start=at, k_start=at, max_q=80, max_k=80)
