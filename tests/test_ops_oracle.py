"""The 64-bit formulas of tests/opscheck.py: their gradients against differences of their values."""
import pytest
import torch

import opscheck as O


def directional(f, x, way, h=1e-5):
    return (f(x + h * way) - f(x - h * way)) / (2 * h)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim, rot", [(8, 8), (12, 6), (16, 0)])
def test_rope_gradient(dim, rot, interleaved):
    g = torch.Generator().manual_seed(dim + rot)
    x, dy, way = (torch.randn(2, 3, 4, dim, generator=g, dtype=O.F64) for _ in range(3))
    w, ww = torch.rand(dim, generator=g, dtype=O.F64) + 0.5, torch.randn(dim, generator=g, dtype=O.F64)
    table = torch.rand(9, rot, generator=g, dtype=O.F64) * 2 - 1
    pos = torch.randint(0, 9, (2, 3), generator=g)
    loss = lambda x, w: (O.rope(x, w, table, pos, 1e-3, interleaved, O.F64)[0] * dy).sum()     # noqa: E731
    dx, _, dw, _ = O.rope_backward(dy, x, w, table, pos, 1e-3, interleaved, O.F64)
    assert abs(directional(lambda t: loss(t, w), x, way) - (dx * way).sum()) < 1e-7
    assert abs(directional(lambda t: loss(x, t), w, ww) - (dw * ww).sum()) < 1e-7


@pytest.mark.parametrize("causal, window, sinks", [(True, 0, 0), (True, 3, 2), (False, 0, 0), (False, 2, 1)])
@pytest.mark.parametrize("nq, nk", [(5, 5), (1, 6), (7, 4), (3, 0)])
def test_attention_gradient(causal, window, sinks, nq, nk):
    g = torch.Generator().manual_seed(nq * 10 + nk)
    q, do = (torch.randn(1, nq, 4, 8, generator=g, dtype=O.F64) for _ in range(2))
    k, v = (torch.randn(1, nk, 2, 8, generator=g, dtype=O.F64) for _ in range(2))
    got = O.attention(q, k, v, do, causal, window, sinks)
    for name, t, fn in (("dq", q, lambda t: (t, k, v)), ("dk", k, lambda t: (q, t, v)), ("dv", v, lambda t: (q, k, t))):
        way = torch.randn(t.shape, generator=g, dtype=O.F64)
        want = directional(lambda t: (O.attention(*fn(t), None, causal, window, sinks)["o"][0] * do).sum(), t, way)
        assert abs(want - (got[name][0] * way).sum()) < 1e-7, name


def test_masks_leave_what_they_say():
    # 4 queries on 6 keys, window 2, one sink: by hand
    rows = O.visible(4, 6, True, 2, 1).int().tolist()
    assert rows == [[1, 1, 1, 0, 0, 0], [1, 0, 1, 1, 0, 0], [1, 0, 0, 1, 1, 0], [1, 0, 0, 0, 1, 1]]
    rows = O.visible(3, 3, False, 2, 1).int().tolist()
    assert rows == [[1, 1, 0], [1, 1, 1], [1, 1, 1]]
    rows = O.visible(3, 2, True, 0, 0).int().tolist()                 # the first query stands before the first key
    assert rows == [[0, 0], [1, 0], [1, 1]]
