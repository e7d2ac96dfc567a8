"""Norms of rows, centred and not, against the 64-bit formulas: every way a row is cut, every type and layout."""
import pytest
import torch

import layercheck as L

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    from paper_2310_09443_amd import ops
    return ops


def make(rows, dim, dtype, wtype=None, weight=True, bias=True, seed=0, off=0.5):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)                                              # noqa: E731
    x = (r(rows, dim) * torch.exp(r(rows, 1)) + off).to(dtype).cuda()
    w = (1 + 0.3 * r(dim)).to(wtype or dtype).cuda() if weight else None
    b = r(dim).to(wtype or dtype).cuda() if bias else None
    return x, w, b, r(rows, dim).to(dtype).cuda()


def check(ops, x, w, b, dy, eps=1e-6, center=True):
    got = {"y": ops.g10_norm(x, w, b, eps, center)}
    assert got["y"].shape == x.shape and got["y"].dtype == x.dtype
    got["dx"], got["dweight"], got["dbias"] = ops.g10_norm_backward(dy, x, w, b, eps, center)
    assert (got["dweight"] is None) == (w is None) and (got["dbias"] is None) == (b is None)
    want = L.norm(x, w, b, eps, center, x.dtype)
    want.update(L.norm(x, w, b, eps, center, x.dtype, dy))
    for n, (y, t) in want.items():
        L.assert_near(got[n].reshape(y.shape), y, t, n)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("center", [False, True])
@pytest.mark.parametrize("dim", [1, 2, 7, 8, 63, 64, 100, 512, 520, 768, 1000, 1024, 1032, 1600, 2048, 2056, 4096, 5001, 8192])
def test_dims(ops, dim, center, dtype):
    check(ops, *make(5, dim, dtype, bias=center, seed=dim), center=center)


@pytest.mark.parametrize("dim", [8200, 16384, 20000, 33333, 65536])
def test_long_rows(ops, dim):
    check(ops, *make(3, dim, torch.bfloat16, seed=dim))
    check(ops, *make(2, dim, torch.float32, seed=dim), center=False)


@pytest.mark.parametrize("rows, dim", [(1, 96), (4, 96), (4099, 40), (9000, 8), (1500, 1032), (700, 9000)])
def test_many_rows(ops, rows, dim):
    """More rows than a backward pass has groups."""
    check(ops, *make(rows, dim, torch.bfloat16, wtype=torch.float32, seed=rows))


def test_weights(ops):
    for dim in (64, 65, 1100):
        for kw in (dict(weight=False), dict(bias=False), dict(weight=False, bias=False), dict(wtype=torch.float32)):
            check(ops, *make(9, dim, torch.float16, **kw))


def test_a_large_mean_leaves_what_is_behind_it(ops):
    """Values of 1000 +- 1: the squares' mean less the mean's square would lose most of the variance in 32 bits."""
    check(ops, *make(6, 512, torch.float32, off=1000.0))


def test_rows_of_one_value(ops):
    x, w, b, dy = make(4, 72, torch.float32)
    x[0], x[1] = 3.25, 0.0
    check(ops, x, w, b, dy, eps=1e-3)
    check(ops, x, w, None, dy, eps=1e-3, center=False)
    x[2, 5] = float("nan")
    y = ops.g10_norm(x, w, b, 1e-3, True)
    assert y[2].isnan().all() and not y[[0, 1, 3]].isnan().any()                             # a row's NaN stays in its row


def test_layouts(ops):
    x, w, b, dy = make(24, 64, torch.bfloat16)
    check(ops, x.view(2, 3, 4, 64), w, b, dy.view(2, 3, 4, 64))
    check(ops, x.view(4, 6, 64).transpose(0, 1), w, b, dy.view(6, 4, 64))
    wide = torch.randn(24, 200, device="cuda").bfloat16()
    check(ops, wide[:, 8:72], w, b, wide[:, 72:136])
    check(ops, wide[:, 5:69], w, b, wide[:, 70:134])
    check(ops, x.t().contiguous().t(), w, b, dy[:1].expand(24, 64))
    check(ops, x, torch.cat([w, w])[1:65], b, dy)
    check(ops, x, torch.stack([w, w], 1)[:, 0], b, dy)
    check(ops, x[0], w, b, dy[0])


def test_no_rows(ops):
    x, w, b, dy = make(4, 72, torch.float32)
    assert ops.g10_norm(x[:0], w, b).shape == (0, 72)
    dx, dw, db = ops.g10_norm_backward(dy[:0], x[:0], w, b)
    assert dx.shape == (0, 72) and not dw.any() and not db.any()


def test_gradients_against_differences(ops):
    """The derivative along a direction, by differences of the formula in 64 bits: their own error is O(h^2)."""
    x, w, b, dy = make(3, 40, torch.float32)
    for t in (x, w, b):
        t.requires_grad_()
    (ops.norm(x, w, b, 1e-5, True) * dy).sum().backward()
    g = torch.Generator().manual_seed(5)

    def f(p):
        c = p[0] - p[0].mean(-1, keepdim=True)
        return float((((c / (c.square().mean(-1, keepdim=True) + L.f32(1e-5)).sqrt()) * p[1] + p[2]) * L.d(dy)).sum())
    p = [L.d(t) for t in (x, w, b)]
    for i, t in enumerate((x, w, b)):
        v, h = torch.randn(p[i].shape, generator=g, dtype=torch.float64), 1e-5
        hi, lo = ([q + (s * h * v if j == i else 0) for j, q in enumerate(p)] for s in (1, -1))
        want = (f(hi) - f(lo)) / (2 * h)
        assert abs(float((L.d(t.grad) * v).sum()) - want) <= 1e-4 * (1 + abs(want))


def test_refusals(ops):
    x, w, b, dy = make(4, 16, torch.float16)
    for bad, match in ((lambda: ops.g10_norm(x.cpu(), w, b), "GPU memory"), (lambda: ops.g10_norm(x.double()), "not supported"), (lambda: ops.g10_norm(x, w[:8]), "weight"),
                       (lambda: ops.g10_norm(x, w, b.float()), "one type"), (lambda: ops.g10_norm(x, w, b, -1.0), "eps"), (lambda: ops.g10_norm(x, w, b, float("inf")), "eps"),
                       (lambda: ops.g10_norm(x, w.bfloat16()), "weight"), (lambda: ops.g10_norm_backward(dy[:2], x, w, b), "dy"),
                       (lambda: ops.g10_norm_backward(dy.float(), x, w, b), "dy"), (lambda: ops.g10_norm(x[:, :0]), "values"),
                       (lambda: ops.g10_norm(torch.zeros(1, 65537, device="cuda")), "65536")):
        with pytest.raises(ValueError, match=match):
            bad()


@pytest.mark.parametrize("dim", [3, 64, 65, 120, 128, 130, 250, 256, 264])
@pytest.mark.parametrize("rows", [1, 7, 8, 31, 33, 1025, 20001])
def test_narrow_rows(ops, rows, dim):
    """Rows side by side in a wavefront, the last one with some of them; more of them than a backward pass has places."""
    check(ops, *make(rows, dim, torch.bfloat16, wtype=torch.float32, seed=rows + dim))
