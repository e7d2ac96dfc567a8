"""The gated MLP's first half and its gradients, against the 64-bit formulas: both layouts of the weights, tiles cut at every edge, every plan."""
import math

import pytest
import torch

import layercheck as L

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    from paper_2310_09443_amd import ops
    return ops


def make(tokens, dim, inner, dtype, out_in=False, seed=0):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)                                              # noqa: E731
    w = [(r(inner, dim) / math.sqrt(dim)).to(dtype).cuda().t() if out_in else (r(dim, inner) / math.sqrt(dim)).to(dtype).cuda() for _ in range(2)]
    return r(tokens, dim).to(dtype).cuda(), w[0], w[1], r(tokens, inner).to(dtype).cuda()


def check(ops, x, gate, up, dh, act="silu"):
    h = ops.g10_gated(x, gate, up, act)
    assert h.shape == dh.shape and h.dtype == x.dtype
    L.assert_gated({"h": h}, L.gated(x, gate, up, act), x.dtype)
    dx, dg, du = ops.g10_gated_backward(dh, x, gate, up, act)
    assert dx.shape == x.shape and dg.shape == gate.shape and du.shape == up.shape
    L.assert_gated(dict(dx=dx, dgate=dg, dup=du), L.gated(x, gate, up, act, dh), x.dtype)
    again = ops.g10_gated_backward(dh, x, gate, up, act)
    assert torch.equal(h, ops.g10_gated(x, gate, up, act)) and all(torch.equal(a, b) for a, b in zip(again, (dx, dg, du)))


@pytest.mark.parametrize("out_in", [False, True])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("tokens, dim, inner", [(1, 8, 8), (1, 64, 128), (7, 72, 136), (32, 64, 128), (33, 128, 256), (64, 200, 8), (65, 8, 264), (130, 264, 392), (257, 136, 520),
                                                (300, 520, 72), (1, 1032, 40), (40, 4104, 16)])
def test_sizes(ops, tokens, dim, inner, dtype, out_in):
    check(ops, *make(tokens, dim, inner, dtype, out_in, seed=tokens + dim))


@pytest.mark.parametrize("out_in", [False, True])
def test_large_tiles(ops, out_in):
    """Enough tiles of 256 rows for a large product, cut at every edge."""
    check(ops, *make(3000, 264, 2056, torch.bfloat16, out_in))
    check(ops, *make(2050, 2056, 1000, torch.float16, out_in), act="gelu")


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_activations(ops, act):
    x, gate, up, dh = make(100, 64, 192, torch.float16)
    check(ops, x * 4, gate, up, dh, act)
    check(ops, x * 0, gate, up, dh, act)
    x[0] = 60.0                                                                              # far out on both sides
    check(ops, x, gate, up, dh * 0.01, act)


@pytest.mark.parametrize("out_in", [False, True])
@pytest.mark.parametrize("tokens, dim, inner", [(5, 1, 1), (9, 7, 13), (33, 65, 100), (2, 1001, 3), (70, 129, 259), (1, 2500, 70), (300, 517, 1030), (1100, 333, 1717)])
def test_odd_sizes(ops, tokens, dim, inner, out_in):
    check(ops, *make(tokens, dim, inner, torch.bfloat16 if dim % 2 else torch.float16, out_in, seed=dim))


def test_layouts(ops):
    x, gate, up, dh = make(24, 64, 128, torch.bfloat16)
    check(ops, x.view(2, 3, 4, 64), gate, up, dh.view(2, 3, 4, 128))
    check(ops, x.view(4, 6, 64).transpose(0, 1), gate, up, dh.view(6, 4, 128))
    wide = torch.randn(24, 300, device="cuda").bfloat16()
    check(ops, wide[:, 8:72], gate, up, wide[:, 104:232])
    check(ops, wide[:, 5:69], gate, up, wide[:, 101:229])
    check(ops, x.t().contiguous().t(), gate, up, dh[:1].expand(24, 128))
    both = torch.cat([gate, up], 1)
    check(ops, x, both[:, :128], both[:, 128:], dh)                                          # halves of one weight
    check(ops, x, gate, both[:, 128:], dh)                                                   # strides that differ
    check(ops, x, gate.t().contiguous().t(), up, dh)                                         # layouts that differ
    check(ops, x, both[:, 1:129], both[:, 3:131], dh)
    check(ops, x[0], gate, up, dh[0])


def test_no_tokens(ops):
    x, gate, up, dh = make(3, 64, 128, torch.bfloat16)
    assert ops.g10_gated(x[:0], gate, up).shape == (0, 128)
    dx, dg, du = ops.g10_gated_backward(dh[:0], x[:0], gate, up)
    assert dx.shape == (0, 64) and not dg.any() and not du.any()


def test_what_lies_behind_the_sizes_is_not_read(ops):
    """NaN around every operand: in the rows' ends that a piece of a tile could reach, in rows behind the last."""
    tokens, dim, inner = 37, 72, 136
    x, gate, up, dh = make(tokens, dim, inner, torch.bfloat16)
    want = ops.g10_gated(x, gate, up), *ops.g10_gated_backward(dh, x, gate, up)

    def around(t):
        big = torch.full((t.shape[0] + 300, t.shape[1] + 304), math.nan, dtype=t.dtype, device="cuda")
        view = big[8:8 + t.shape[0], 16:16 + t.shape[1]]
        view.copy_(t)
        return view
    a = [around(t) for t in (x, gate, up, dh)]
    got = ops.g10_gated(*a[:3]), *ops.g10_gated_backward(a[3], *a[:3])
    for g, w in zip(got, want):
        assert torch.equal(g, w)


def test_gradients_against_differences(ops):
    """Along a direction, by differences of the formula in 64 bits.  Each value of a gradient is off by two roundings at most, independent ones, so
    that their sum along v is off by 2 u |grad| |v| at most."""
    x, gate, up, dh = make(20, 64, 128, torch.float16)
    leaves = [t.detach().clone().requires_grad_() for t in (x, gate, up)]
    for act in ("silu", "gelu"):
        for t in leaves:
            t.grad = None
        (ops.gated(*leaves, act) * dh).sum().backward()
        p = [L.d(t) for t in leaves]

        def f(q):
            g = q[0] @ q[1]
            s = torch.sigmoid(g) if act == "silu" else torch.special.ndtr(g)
            return float((g * s * (q[0] @ q[2]) * L.d(dh)).sum())
        gen = torch.Generator().manual_seed(5)
        for i, t in enumerate(leaves):
            v, h = torch.randn(p[i].shape, generator=gen, dtype=torch.float64), 1e-5
            hi, lo = ([q + (s * h * v if j == i else 0) for j, q in enumerate(p)] for s in (1, -1))
            want, got = (f(hi) - f(lo)) / (2 * h), float((L.d(t.grad) * v).sum())
            assert abs(got - want) <= 2 * L.u(torch.float16) * float(L.d(t.grad).norm() * v.norm()) + 1e-4


def test_values_that_are_no_numbers_stay_in_their_rows(ops):
    x, gate, up, dh = make(70, 64, 128, torch.bfloat16)
    x[3, 5] = math.nan
    h = ops.g10_gated(x, gate, up)
    assert h[3].isnan().all() and not h[:3].isnan().any() and not h[4:].isnan().any()


def test_refusals(ops):
    x, gate, up, dh = make(4, 16, 24, torch.float16)
    for bad, match in ((lambda: ops.g10_gated(x.cpu(), gate, up), "GPU memory"), (lambda: ops.g10_gated(x.float(), gate.float(), up.float()), "not supported"),
                       (lambda: ops.g10_gated(x, gate[:8], up), "gate"), (lambda: ops.g10_gated(x, gate, up[:, :8]), "up"), (lambda: ops.g10_gated(x, gate, up, "relu"), "act"),
                       (lambda: ops.g10_gated(x, gate.bfloat16(), up), "gate"), (lambda: ops.g10_gated_backward(dh[:2], x, gate, up), "dh"),
                       (lambda: ops.g10_gated_backward(dh.float(), x, gate, up), "dh"), (lambda: ops.g10_gated(x, gate[:, :0], up[:, :0]), "gate")):
        with pytest.raises(ValueError, match=match):
            bad()
