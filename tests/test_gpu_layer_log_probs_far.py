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
