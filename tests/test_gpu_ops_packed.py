"""Packed sequences in a buffer that is longer than they are: rows before the first and behind the last one belong to none, and come out as
what sees nothing, whatever the memory of the outputs held."""
import pytest
import torch

import opscheck as O

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    from paper_2310_09443_amd import ops
    return ops


def dirty(*like):
    """Leaves NaN in the memory that the next tensors of these sizes are made of."""
    held = [torch.full_like(t, float("nan")) for t in like for _ in range(4)]
    torch.cuda.synchronize()
    del held


# one head group; lengths that take the kernel for few queries (whole blocks, shares), the one for many, keys' gradients by tiles and in shares
@pytest.mark.parametrize("dim, dtype", [(64, torch.float16), (128, torch.bfloat16), (40, torch.bfloat16)])
@pytest.mark.parametrize("nq, nk, heads, lead, tail", [
    ([37, 50], [37, 50], 2, 3, 38), ([0, 1, 1], [5, 9, 0], 4, 2, 1), ([1, 2], [2000, 900], 4, 0, 700), ([200, 0, 300], [200, 70, 300], 4, 130, 0),
    ([640, 500], [640, 500], 16, 1, 4000), ([0, 0], [0, 0], 2, 4, 60)])
def test_rows_of_no_sequence(ops, nq, nk, heads, lead, tail, dim, dtype):
    at = [(lead + torch.tensor([0] + n).cumsum(0)).to(torch.int32) for n in (nq, nk)]
    rows = [int(a[-1]) + tail for a in at]
    g = torch.Generator().manual_seed(dim + sum(nq))
    q, do = (torch.randn(rows[0], heads, dim, generator=g).to(dtype).cuda() for _ in range(2))
    k, v = (torch.randn(rows[1], heads // 2, dim, generator=g).to(dtype).cuda() for _ in range(2))
    want = O.attention(q.cpu(), k.cpu(), v.cpu(), do.cpu(), True, 0, 0, q_start=at[0], k_start=at[1])
    for t, a in ((q, at[0]), (do, at[0]), (k, at[1]), (v, at[1])):     # what such rows hold is not read
        t[:a[0]] = t[a[-1]:] = float("nan")
    args = dict(q_start=at[0].cuda(), k_start=at[1].cuda())
    lse = torch.empty(heads, rows[0], device="cuda")
    dirty(q, lse)
    o, lse = ops.g10_attention(q, k, v, **args)
    dirty(q, k, v)
    got = dict(zip(("o", "dq", "dk", "dv"), (o, *ops.g10_attention_backward(do, q, k, v, o, lse, **args))))
    for n, x in got.items():
        O.assert_near(x, *want[n], n)
        a = at[0] if n in ("o", "dq") else at[1]
        assert not x[:a[0]].any() and not x[a[-1]:].any(), n
    a, value = at[0], torch.full_like(lse, -float("inf"))
    assert torch.equal(lse[:, :a[0]], value[:, :a[0]]) and torch.equal(lse[:, a[-1]:], value[:, a[-1]:])
    O.assert_near(lse[:, a[0]:a[-1]], *(t[:, a[0]:a[-1]] for t in want["lse"]), "lse")


def test_rows_and_no_sequence(ops):
    q = torch.randn(5, 2, 64, device="cuda").bfloat16()
    at = torch.zeros(1, dtype=torch.int32, device="cuda")
    dirty(q, torch.empty(2, 5, device="cuda"))
    o, lse = ops.g10_attention(q, q, q, q_start=at, k_start=at)
    assert not o.any() and (lse == -float("inf")).all()
    assert not any(x.any() for x in ops.g10_attention_backward(q, q, q, q, o, lse, q_start=at, k_start=at))


def test_a_projection_learns_from_its_sequences_only(ops):
    """The gradient of a weight before the attention, x^T dq and the like, takes nothing from the padding."""
    g = torch.Generator().manual_seed(3)
    x, w = torch.randn(128, 64, generator=g).bfloat16().cuda(), (torch.randn(64, 3 * 64, generator=g) / 8).bfloat16().cuda()
    at = torch.tensor([0, 40, 90], dtype=torch.int32, device="cuda")
    grads = []
    for rows in (128, 90):
        weight = w.clone().requires_grad_()
        q, k, v = (x[:rows] @ weight).view(rows, 3, 1, 64).unbind(1)
        dirty(q, q)
        o = ops.attention(q, k, v, q_start=at, k_start=at)
        dirty(q, q)
        (o.float().square().sum()).backward()
        grads.append(weight.grad)
    # the library's products of 128 and of 90 rows may be summed in other orders: each is rounded to bfloat16, q, k and v as well
    assert (grads[0] - grads[1]).abs().max() <= 2.0 ** -6 * grads[1].abs().max()


def test_many_sequences_whose_lengths_are_not_told(ops):
    """One token each: the output is its value, the value's gradient the sum over its heads.  A grid for the longest possible sequence
    would have 2^32 workgroups."""
    n, heads, kv, dim = 65600, 32, 8, 8
    g = torch.Generator().manual_seed(7)
    q, do = (torch.randn(n, heads, dim, generator=g).bfloat16().cuda() for _ in range(2))
    k, v = (torch.randn(n, kv, dim, generator=g).bfloat16().cuda() for _ in range(2))
    at = torch.arange(n + 1, dtype=torch.int32, device="cuda")
    dirty(q)
    o, lse = ops.g10_attention(q, k, v, q_start=at, k_start=at)
    assert torch.equal(o, v.repeat_interleave(heads // kv, 1))
    score = (O.d(q) * O.d(k).repeat_interleave(heads // kv, 1))
    O.assert_near(lse, score.sum(-1).t() * dim ** -0.5, ((dim + 12) * O.U32 * (score.abs().sum(-1).t() * dim ** -0.5 + 1)), "lse")
    dirty(k)
    dv = ops.g10_attention_backward(do, q, k, v, o, lse, q_start=at, k_start=at)[2]
    want = O.d(do).view(n, kv, heads // kv, dim)
    # P is 2^(score - lse), both in 32 bits
    O.assert_near(dv, want.sum(2), O.rounding(want.sum(2), torch.bfloat16) + (2 * (dim + 12) * 8 + 8) * O.U32 * want.abs().sum(2), "dv")
