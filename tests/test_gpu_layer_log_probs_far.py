"""Log probabilities of rows far from zero: an offset that all logits have in common, rows masked as a whole, logits at the type's end.  What counts is how
far a logit lies from the row's largest."""
import math

import pytest
import torch

import logpcheck as K

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.float16, torch.bfloat16]


@pytest.fixture(scope="module")
def ops():
    from paper_2310_09443_amd import ops
    return ops


def forward(ops, x, t, top, scale):
    logp, lse, ent, top_logp, ids = ops.g10_log_probs(x, t, entropy=True, top=top, scale=scale)
    return dict(logp=logp, lse=lse, entropy=ent, top_logp=top_logp), ids


def ends(dtype):
    """Logits that a whole row may be set to."""
    f = torch.finfo(dtype)
    return [v for v in (f.min, f.max, -1e9, 1e9, -1e6, 3e4, -3e4, -0.0) if abs(v) <= f.max]


@pytest.mark.parametrize("scale", [0.5, 1.0, 1.25])
@pytest.mark.parametrize("vocab", [5, 1003, 32000, 70000])
@pytest.mark.parametrize("dtype", TYPES)
def test_rows_all_alike(ops, dtype, vocab, scale):
    """-log V each, wherever the row lies.  A sum of V equal exponentials is off by one rounding for each addition; an exponential, the logarithm, difference and
    product by two each, of log V and of up to 6 that the maximum's own rounding puts in.  In the entropy the sum of e d is divided by the sum of e, both
    off so, and d is up to 4: the maximum's rounding."""
    values = ends(dtype)
    x = torch.tensor(values, dtype=dtype, device="cuda")[:, None].repeat(1, vocab)
    t = torch.arange(len(values), device="cuda") % vocab
    got, ids = forward(ops, x, t, 4, scale)
    want, rest = -math.log(vocab), 8 * math.log(vocab) + 48
    for y, n in ((got["logp"], 1), (got["top_logp"], 1), (-got["entropy"], 9)):
        assert ((y.double() - want).abs() <= K.U32 * (n * K.additions(vocab) + rest)).all(), y
    assert (ids == torch.arange(4, device="cuda")).all()
    K.check(dict(lse=got["lse"]), K.log_probs(x, t, scale)[0])


@pytest.mark.parametrize("offset", [0.0, 40.0, -3e3, 1e4, 1e6, -3e7])
@pytest.mark.parametrize("vocab", [300, 5003, 30522, 100001])
def test_a_common_offset(ops, vocab, offset):
    x = (torch.randn(6, vocab, generator=torch.Generator().manual_seed(vocab)) * 3 + offset).cuda()
    t = torch.randint(0, vocab, (6,), generator=torch.Generator().manual_seed(1)).cuda()
    for scale in (1.0, 0.7):
        got, ids = forward(ops, x, t, 9, scale)
        want, wids = K.log_probs(x, t, scale, top=9)
        K.check(got, want)
        assert torch.equal(ids.cpu(), wids)


def mixed(dtype, vocab):
    """Rows in which far logits and near ones meet, in every part of a long row and in some."""
    low, high = torch.finfo(dtype).min, torch.finfo(dtype).max
    x = (torch.randn(17, vocab, generator=torch.Generator().manual_seed(vocab)) * 2).to(dtype).cuda()
    x[0, ::2], x[1, 5:], x[2, : vocab // 2] = low, low, low
    x[3], x[3, vocab // 3] = low, 1.0
    x[4], x[4, -1] = high, low
    x[5], x[5, :-2] = high, 0.0
    x[6, ::3] = -math.inf
    x[7] = -math.inf
    x[8], x[8, 3:] = low, -math.inf
    x[9, : vocab // 2] = low / 2
    x[10], x[10, 1] = high, high / 2
    return x


@pytest.mark.parametrize("scale", [0.25, 1.0, 1.25])
@pytest.mark.parametrize("vocab", [40, 2050, 9000, 70000])
@pytest.mark.parametrize("dtype", TYPES)
def test_far_and_near_in_a_row(ops, dtype, vocab, scale):
    x = mixed(dtype, vocab)
    for at in (0, 1, 5, vocab // 2, vocab - 1):
        t = torch.full((17,), at, device="cuda")
        got, ids = forward(ops, x, t, 7, scale)
        want, wids = K.log_probs(x, t, scale, top=7)
        K.check(got, want)
        assert torch.equal(ids.cpu(), wids)


@pytest.mark.parametrize("rows, vocab", [(2, 400000), (3, 65536), (70, 131072), (600, 20000)])
@pytest.mark.parametrize("dtype", TYPES)
def test_no_logit_is_lost_from_the_sums(ops, rows, vocab, dtype):
    """Ordinary rows, to what a thread's additions leave: a part's last values would be seen."""
    x = (torch.randn(rows, vocab, generator=torch.Generator().manual_seed(rows)) * 2).to(dtype).cuda()
    t = torch.randint(0, vocab, (rows,), generator=torch.Generator().manual_seed(1)).cuda()
    got, _ = forward(ops, x, t, 3, 1.0)
    K.check(got, K.log_probs(x, t, 1.0, top=3)[0])


# -------------------------------------------------------------------------------------------------------------- gradients
NEAR = {torch.float32: 64.0, torch.float16: 256.0, torch.bfloat16: 256.0}                   # lse up to which p is taken from it


def both(ops, x, t, dl, de, scale):
    _, lse, ent, _, _ = ops.g10_log_probs(x, t, entropy=True, scale=scale)
    K.check(dict(dlogits=ops.g10_log_probs_backward(dl, x, t, lse, de, ent, scale)), K.log_probs(x, t, scale, dlogp=dl, dentropy=de, near=NEAR[x.dtype])[0])


def shares(rows):
    g = torch.Generator().manual_seed(rows)
    return [torch.randn(rows, generator=g).cuda() for _ in range(2)]


@pytest.mark.parametrize("scale", [0.5, 1.0, 1.25])
@pytest.mark.parametrize("vocab", [5, 1003, 32000, 70000])
@pytest.mark.parametrize("dtype", TYPES)
def test_gradients_of_rows_all_alike(ops, dtype, vocab, scale):
    """scale dlogp ([j = t] - 1 / V), and nothing of the entropy, which is as large as it can be.  A probability is off by the sum's additions and by
    some twenty roundings of log V (of lse, of its two products, of the argument) and of 1; then the result's own."""
    values = ends(dtype)
    x = torch.tensor(values, dtype=dtype, device="cuda")[:, None].repeat(1, vocab)
    t = torch.arange(len(values), device="cuda") % vocab
    dl, de = shares(len(values))
    _, lse, _, _, _ = ops.g10_log_probs(x, t, scale=scale)
    got = ops.g10_log_probs_backward(dl, x, t, lse, scale=scale).double()
    want = -dl.double()[:, None].expand(-1, vocab) / vocab * scale
    want = want.scatter_add(1, t[:, None], dl.double()[:, None] * scale)
    off = (K.additions(vocab) + 20 * math.log(vocab) + 60) * K.U32
    assert ((got - want).abs() <= K.rounding(want.cpu(), dtype).cuda() + off * want.abs()).all()
    both(ops, x, t, dl, None, scale)
    both(ops, x, t, dl, de, scale)


@pytest.mark.parametrize("offset", [0.0, 40.0, 70.0, -3e3, 1e4, 1e6, -3e7])
@pytest.mark.parametrize("vocab", [300, 5003, 30522, 100001])
def test_gradients_with_a_common_offset(ops, vocab, offset):
    x = (torch.randn(6, vocab, generator=torch.Generator().manual_seed(vocab)) * 3 + offset).cuda()
    t = torch.randint(0, vocab, (6,), generator=torch.Generator().manual_seed(1)).cuda()
    for scale in (1.0, 0.7):
        both(ops, x, t, *shares(6), scale)
    if abs(offset) < 1e5:
        both(ops, x.half(), t, *shares(6), 1.0)
        both(ops, x.bfloat16(), t, *shares(6), 1.0)


@pytest.mark.parametrize("scale", [0.25, 1.0, 1.25])
@pytest.mark.parametrize("vocab", [40, 2050, 9000, 70000])
@pytest.mark.parametrize("dtype", TYPES)
def test_gradients_of_far_and_near_in_a_row(ops, dtype, vocab, scale):
    x = mixed(dtype, vocab)
    for at in (0, vocab // 2, vocab - 1):
        t = torch.full((17,), at, device="cuda")
        both(ops, x, t, shares(17)[0], None, scale)
        both(ops, x, t, *shares(17), scale)


@pytest.mark.parametrize("rows, vocab", [(1, 400000), (300, 70000), (2047, 16400), (2048, 16400)])
def test_gradients_of_far_rows_in_parts_and_whole(ops, rows, vocab):
    x = (torch.randn(rows, vocab, generator=torch.Generator().manual_seed(rows)) * 2).cuda()
    x[::2] += 1e5
    t = torch.randint(0, vocab, (rows,), generator=torch.Generator().manual_seed(1)).cuda()
    dl, de = shares(rows)
    _, lse, ent, _, _ = ops.g10_log_probs(x, t, entropy=True)
    got = ops.g10_log_probs_backward(dl, x, t, lse, de, ent)
    for a in range(0, rows, 64):                                                             # (64 bits of them all are 1 GB)
        at = slice(a, min(a + 8, rows))
        K.check(dict(dlogits=got[at]), K.log_probs(x[at], t[at], 1.0, dlogp=dl[at], dentropy=de[at], near=64.0)[0])


@pytest.mark.parametrize("rows, vocab", [(3, 40), (2, 100000), (40, 20001), (600, 9000)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gradients_over_the_logits(ops, rows, vocab, dtype):
    """Far rows and near ones, written where the logits lay: a row is summed again from logits, not from gradients."""
    import ctypes as C
    x = (torch.randn(rows, vocab, generator=torch.Generator().manual_seed(rows)) * 2).to(dtype).cuda()
    x[::2] += 3e4
    t = torch.randint(0, vocab, (rows,), generator=torch.Generator().manual_seed(1)).cuda()
    dl, de = shares(rows)
    _, lse, ent, _, _ = ops.g10_log_probs(x, t, entropy=True)
    want, z = K.log_probs(x, t, 1.0, dlogp=dl, dentropy=de, near=NEAR[dtype])[0], x.clone()
    q = ops._LogProbs(logits=z.data_ptr(), tokens=t.data_ptr(), lse=lse.data_ptr(), entropy=ent.data_ptr(), dlogp=dl.data_ptr(), dentropy=de.data_ptr(), dlogits=z.data_ptr(),
                      logits_stride=vocab, dlogits_stride=vocab, rows=rows, vocab=vocab, scale=1.0, ignore=-100, type=ops._TYPE[dtype])
    assert ops._load().g10_log_probs_backward(C.byref(q), torch.cuda.current_stream().cuda_stream) == 0
    K.check(dict(dlogits=z), want)
