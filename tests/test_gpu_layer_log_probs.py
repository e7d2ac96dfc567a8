"""Log probabilities, entropy, the likeliest tokens and the logits' gradient, against the 64-bit formulas."""
import math

import pytest
import torch

import layercheck as L

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    from paper_2310_09443_amd import ops
    return ops


def make(rows, vocab, dtype, seed=0, spread=2.0):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(rows, vocab, generator=g) * spread).to(dtype).cuda()
    t = torch.randint(0, vocab, (rows,), generator=g).cuda()
    return x, t, torch.randn(rows, generator=g).cuda(), torch.randn(rows, generator=g).cuda()


def check(ops, x, t, dl=None, de=None, top=0, scale=1.0, ignore=-100):
    logp, lse, ent, top_logp, top_ids = ops.g10_log_probs(x, t, entropy=True, top=top, scale=scale, ignore=ignore)
    got = dict(logp=logp, lse=lse, entropy=ent, top_logp=top_logp)
    if dl is not None or de is not None:
        got["dlogits"] = ops.g10_log_probs_backward(dl, x, t, lse, de, ent, scale, ignore)
        assert got["dlogits"].shape == x.shape and got["dlogits"].dtype == x.dtype
    want, ids = L.log_probs(x, t, scale, ignore, top, dl, de)
    for n, (y, tol) in want.items():
        L.assert_near(got[n].reshape(y.shape), y, tol, n)
    if top:
        assert torch.equal(top_ids.cpu().reshape(ids.shape), ids)
    assert (logp is None) == (t is None) and (top_ids is None) == (not top)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("vocab", [1, 2, 5, 8, 63, 64, 100, 257, 1000, 2047, 4096, 4097, 5003, 32000])
def test_vocabularies(ops, vocab, dtype):
    x, t, dl, de = make(5, vocab, dtype, seed=vocab)
    check(ops, x, t, dl, de, top=min(vocab, 7))
    check(ops, x, t, dl, None, scale=0.7)
    check(ops, x, None, None, de, top=min(vocab, 64), scale=1.7)


@pytest.mark.parametrize("rows, vocab", [(1, 200000), (3, 50001), (600, 5000), (513, 30522), (70000, 9)])
def test_rows(ops, rows, vocab):
    x, t, dl, de = make(rows, vocab, torch.bfloat16 if rows < 600 else torch.float32, seed=rows)
    check(ops, x, t, dl, de, top=5)


@pytest.mark.parametrize("rows, vocab", [(1, 65536), (1, 400000), (3, 100001), (64, 70000), (65, 70000), (17, 131072)])
def test_rows_in_parts(ops, rows, vocab):
    """Few long rows are cut and joined: each kind of row that can go wrong in one part alone or in all."""
    for dtype in (torch.bfloat16, torch.float32):
        x, t, dl, de = make(rows, vocab, dtype, seed=vocab)
        low = torch.finfo(dtype).min
        if rows >= 17:
            x[0], x[1] = -math.inf, low
            x[2, :-5], x[3, 5:], x[4] = -math.inf, -math.inf, 0.25                                # one part has something, all are alike
            x[5, : vocab // 2] = low
            x[6, ::2] = low
            x[7] = torch.arange(vocab, device="cuda").div(vocab // 8, rounding_mode="floor").to(dtype)
        check(ops, x, t, dl, de, top=20)
        check(ops, x, t, dl, None, top=64, scale=0.6)
        check(ops, x, None, None, de, top=1)
        check(ops, x, t, dl, de)
        if rows >= 17:
            x[9, vocab - 2], x[10, 3], x[11] = math.nan, math.inf, math.nan
            logp, lse, ent, top_logp, ids = ops.g10_log_probs(x, t, entropy=True, top=5)
            for y in (logp, lse, ent, top_logp):
                assert y[9:12].isnan().all() and not y[12:].isnan().any()
            assert ids[9, 0] == vocab - 2 and ids[10, 0] == 3 and ids[11].tolist() == [0, 1, 2, 3, 4]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_equal_logits_come_in_their_own_order(ops, dtype):
    x, t, _, _ = make(6, 9000, dtype)
    x[0] = 0.25                                                                              # all alike
    x[1] = x[1].round()                                                                      # many alike
    x[2, ::3], x[2, 1::3] = 0.0, -0.0                                                        # zeros of both signs are equal
    x[3] = torch.arange(9000, device="cuda").div(1000, rounding_mode="floor").to(dtype)      # rising: the last thousand is the top
    x[4] = -x[3]
    for top in (1, 20, 64):
        check(ops, x, t, top=top)
        check(ops, x[:, :801], t.clamp(max=800), top=top)


def test_more_candidates_than_there_is_room_for(ops):
    """One thread's values are the row's largest: every eighth-of-a-thousandth piece of 16 bytes, which the same threads read."""
    for dtype, n in ((torch.bfloat16, 8), (torch.float32, 4)):
        x, t, _, _ = make(3, 400000, dtype, seed=4)
        piece = torch.arange(400000 // n, device="cuda")
        hot = (piece % 1024 < 40).repeat_interleave(n)                                       # 40 of 1024 threads' pieces
        x[:, hot] += 100
        check(ops, x, t, top=64)
        x, t, _, _ = make(600, 30000, dtype, seed=5)
        hot = (torch.arange(30000 // n, device="cuda") % 256 < 30).repeat_interleave(n)
        x[:, hot] += 100
        check(ops, x, t, top=20)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
def test_masked_places(ops, dtype):
    x, t, dl, de = make(8, 1003, dtype)
    low = torch.finfo(dtype).min
    x[0] = -math.inf                                                                         # nothing is left
    x[1, :] = -math.inf
    x[1, 77] = 3.0                                                                           # one place
    x[2, 500:] = -math.inf
    x[3, ::2] = low                                                                          # masked with the type's lowest value
    x[4] = low
    x[5, :990] = -math.inf                                                                   # the first values a thread sees are none
    t[1], t[2] = 77, 700                                                                     # (a token without probability: -inf)
    check(ops, x, t, dl, de, top=10)
    check(ops, x, t, dl, None, top=64, scale=0.5)


def test_values_that_are_no_numbers(ops):
    x, t, dl, de = make(6, 3000, torch.float32)
    x[0, 100], x[1, 5], x[2] = math.nan, math.inf, math.nan
    x[3, 2999] = -math.nan
    logp, lse, ent, top_logp, ids = ops.g10_log_probs(x, t, entropy=True, top=5)
    g = ops.g10_log_probs_backward(dl, x, t, lse, de, ent)
    for y in (logp, lse, ent, top_logp, g):
        assert y[:4].isnan().all() and not y[4:].isnan().any()
    assert ids[0, 0] == 100 and ids[1, 0] == 5 and ids[2].tolist() == [0, 1, 2, 3, 4] and ids[3, 0] == 2999
    assert (ids >= 0).all() and (ids < 3000).all()
    check(ops, x[4:], t[4:], dl[4:], de[4:], top=5)


def test_tokens(ops):
    x, t, dl, de = make(9, 500, torch.bfloat16)
    t[0], t[1], t[2], t[3] = -100, 500, -1, 2 ** 40
    check(ops, x, t, dl, None)
    check(ops, x, t, dl, de)
    check(ops, x, t, dl, de, ignore=500)
    check(ops, x, t.clamp(0, 499).int(), dl, de, ignore=3)
    dl[5] = 0.0
    x[5, 3] = math.nan                                                                       # a row that has no share in the loss
    x[0, 3] = math.nan
    logp, lse, _, _, _ = ops.g10_log_probs(x, t)
    g = ops.g10_log_probs_backward(dl, x, t, lse)
    assert not g[0].any() and not g[5].any() and g[1:4].isnan().all()


def test_layouts(ops):
    x, t, dl, de = make(24, 130, torch.bfloat16)
    check(ops, x.view(2, 3, 4, 130), t.view(2, 3, 4), dl.view(2, 3, 4), de.view(2, 3, 4), top=3)
    check(ops, x.view(4, 6, 130).transpose(0, 1), t.view(6, 4), dl.view(6, 4), None, top=3)
    for dtype in (torch.bfloat16, torch.float32):
        wide = torch.randn(24, 301, device="cuda").to(dtype)                                 # rows at every place within 16 bytes
        check(ops, wide[:, :301], t, dl, de, top=3)
        check(ops, wide[:, 7:137], t, dl, de, top=3)
        check(ops, wide[:, 8:9], torch.zeros_like(t), dl, de, top=1)
    check(ops, x.t().contiguous().t(), t, dl, de, top=2)
    check(ops, x[:1].expand(24, 130), t, dl, de, top=2)
    check(ops, x[0], t[0], dl[0], de[0], top=2)
    check(ops, x, torch.stack([t, t], 1)[:, 0], torch.stack([dl, dl], 1)[:, 1], de, top=2)


def test_no_rows(ops):
    x, t, dl, de = make(4, 60, torch.float32)
    logp, lse, ent, top_logp, ids = ops.g10_log_probs(x[:0], t[:0], entropy=True, top=4)
    assert logp.shape == lse.shape == ent.shape == (0,) and top_logp.shape == ids.shape == (0, 4)
    assert ops.g10_log_probs_backward(dl[:0], x[:0], t[:0], lse).shape == (0, 60)


def test_gradients_through_autograd_and_against_differences(ops):
    x, t, dl, de = make(4, 50, torch.float32)
    x.requires_grad_()
    logp, ent = ops.log_probs(x, t, entropy=True, scale=1.3)
    ((logp * dl).sum() + (ent * de).sum()).backward()
    want, _ = L.log_probs(x, t, 1.3, -100, 0, dl, de)
    L.assert_near(x.grad, *want["dlogits"], "dlogits")
    v = torch.randn(4, 50, generator=torch.Generator().manual_seed(3), dtype=torch.float64)

    def f(y):
        a = torch.log_softmax(y * L.f32(1.3), -1)
        return float((a.gather(1, t.cpu()[:, None])[:, 0] * L.d(dl)).sum() - ((a.exp() * a).sum(-1) * L.d(de)).sum())
    h = 1e-5
    diff = (f(L.d(x) + h * v) - f(L.d(x) - h * v)) / (2 * h)
    assert abs(float((L.d(x.grad) * v).sum()) - diff) <= 1e-4 * (1 + abs(diff))
    x.grad = None
    ops.log_probs(x, t).sum().backward()                                                     # one output alone
    want, _ = L.log_probs(x, t, 1.0, -100, 0, torch.ones(4), None)
    L.assert_near(x.grad, *want["dlogits"], "dlogits")


def test_refusals(ops):
    x, t, dl, de = make(4, 60, torch.float16)
    lse = dl
    for bad, match in ((lambda: ops.g10_log_probs(x.cpu(), t), "GPU memory"), (lambda: ops.g10_log_probs(x, t.float()), "int64"),
                       (lambda: ops.g10_log_probs(x, t[:3]), "one for each row"), (lambda: ops.g10_log_probs(x, t, top=61), "top"),
                       (lambda: ops.g10_log_probs(x.repeat(1, 2), t, top=65), "top"), (lambda: ops.g10_log_probs(x, t, top=-1), "top"),
                       (lambda: ops.g10_log_probs(x, t, scale=0.0), "scale"), (lambda: ops.g10_log_probs(x, t, scale=math.nan), "scale"),
                       (lambda: ops.g10_log_probs(x[:, :0], t), "values"), (lambda: ops.g10_log_probs(x.long(), t), "not supported"),
                       (lambda: ops.g10_log_probs_backward(dl, x, None, lse), "without tokens"), (lambda: ops.g10_log_probs_backward(dl, x, t, lse, de), "entropy"),
                       (lambda: ops.g10_log_probs_backward(dl.half(), x, t, lse), "dlogp"), (lambda: ops.g10_log_probs_backward(dl, x, t, lse[:2]), "lse")):
        with pytest.raises(ValueError, match=match):
            bad()
