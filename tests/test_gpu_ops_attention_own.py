"""How exact a sequence's gradients are goes by its own lengths, whatever its neighbours', and a query's by the keys that it sees."""
import pytest
import torch

import opscheck as O

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    from paper_2310_09443_amd import ops
    return ops


def make(lead_q, lead_k, heads, kv, dim, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)                                          # noqa: E731
    return [t.cuda() for t in ((r(*lead_q, heads, dim) * 1.5).to(dtype), r(*lead_k, kv, dim).to(dtype), r(*lead_k, kv, dim).to(dtype), r(*lead_q, heads, dim).to(dtype))]


def times_one_rounding(got, exact, dtype):
    """Error as a multiple of what one rounding leaves."""
    return float((O.d(got) - exact).norm() / (exact.to(dtype).double() - exact).norm())


# both halves of the 16-bit factors: their own rounding, and up to a quarter of it beside (single factors: 1.41 and more)
BOTH = 1.25


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dim, causal, window", [(64, True, 0), (128, True, 0), (128, False, 0), (64, False, 0), (128, True, 900)])
def test_short_sequences_beside_long_ones(ops, dim, causal, window, dtype):
    n = [7, 1900, 60, 0, 120, 1500, 700, 30]
    at = torch.tensor([0] + n).cumsum(0).to(torch.int32)
    q, k, v, do = make((sum(n),), (sum(n),), 4, 2, dim, dtype, dim)
    args = dict(causal=causal, window=window)
    want = O.attention(q.cpu(), k.cpu(), v.cpu(), do.cpu(), causal, window, 0, q_start=at, k_start=at)
    o, lse = ops.g10_attention(q, k, v, q_start=at.cuda(), k_start=at.cuda(), **args)
    got = dict(zip(("dq", "dk", "dv"), ops.g10_attention_backward(do, q, k, v, o, lse, q_start=at.cuda(), k_start=at.cuda(), **args)))
    for name, x in got.items():
        O.assert_near(x, *want[name], name)
        for i, m in enumerate(n):
            if 0 < m <= (768 if name == "dq" else 128):
                s = slice(int(at[i]), int(at[i + 1]))
                assert times_one_rounding(x[s], want[name][0][s], dtype) <= BOTH, (name, m)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dim", [64, 128])
def test_short_ones_by_k_len(ops, dim, dtype):
    q, k, v, do = make((4, 900), (4, 900), 2, 2, dim, dtype, dim)
    k_len = torch.tensor([900, 100, 0, 500], dtype=torch.int32)
    want = O.attention(q.cpu(), k.cpu(), v.cpu(), do.cpu(), False, 0, 0, k_len=k_len)
    o, lse = ops.g10_attention(q, k, v, causal=False, k_len=k_len.cuda())
    for name, x in zip(("dq", "dk", "dv"), ops.g10_attention_backward(do, q, k, v, o, lse, causal=False, k_len=k_len.cuda())):
        O.assert_near(x, *want[name], name)
        for b in (1, 3) if name == "dq" else (1,):
            assert times_one_rounding(x[b], want[name][0][b], dtype) <= BOTH, (name, b)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("nq, nk, causal, window, sinks", [(1500, 1500, True, 0, 0), (1500, 1500, True, 1000, 4), (1300, 1500, False, 700, 30), (1500, 1000, False, 900, 0)])
def test_queries_that_see_few_keys_of_many(ops, nq, nk, causal, window, sinks, dtype):
    q, k, v, do = make((1, nq), (1, nk), 4, 2, 128, dtype, nk)
    args = dict(causal=causal, window=window, sinks=sinks)
    want = O.attention(q.cpu(), k.cpu(), v.cpu(), do.cpu(), causal, window, sinks)
    o, lse = ops.g10_attention(q, k, v, **args)
    got = dict(zip(("dq", "dk", "dv"), ops.g10_attention_backward(do, q, k, v, o, lse, **args)))
    for name, x in got.items():
        O.assert_near(x, *want[name], name)
    keys = O.visible(nq, nk, causal, window, sinks).sum(1)
    few = (keys > 0) & (keys <= 768)
    assert few.any()
    assert times_one_rounding(got["dq"][:, few.cuda()], want["dq"][0][:, few], dtype) <= BOTH
    # packed between others, from the same forward pass, it is the same number for number: what decides is its own
    at = [torch.tensor([0, 9, 9 + m, 14 + m], dtype=torch.int32, device="cuda") for m in (nq, nk)]
    wrap = lambda t: torch.cat([t[0, :9], t[0], t[0, :5]])                               # noqa: E731
    all_lse = torch.cat([lse[0, :, :9], lse[0], lse[0, :, :5]], 1)
    dq = ops.g10_attention_backward(wrap(do), wrap(q), wrap(k), wrap(v), wrap(o), all_lse, q_start=at[0], k_start=at[1], **args)[0]
    assert torch.equal(dq[9:9 + nq], got["dq"][0])
