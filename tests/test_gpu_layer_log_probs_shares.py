"""The gradient of rows that have no share in a loss: nothing, whatever the row holds and whatever came of it forward."""
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


def make(rows, vocab, dtype):
    g = torch.Generator().manual_seed(vocab)
    x = (torch.randn(rows, vocab, generator=g) * 2).to(dtype).cuda()
    return x, torch.randint(0, vocab, (rows,), generator=g).cuda(), torch.randn(rows, generator=g).cuda(), torch.randn(rows, generator=g).cuda()


@pytest.mark.parametrize("vocab", [60, 3001, 70000])
@pytest.mark.parametrize("dtype", TYPES)
def test_no_share_of_entropy_in_rows_that_have_none(ops, dtype, vocab):
    """Entropy NaN and its share 0, as autograd hands it over where the loss goes by the tokens alone."""
    x, t, dl, de = make(6, vocab, dtype)
    x[0, 3], x[1, 4], x[2] = math.nan, math.inf, math.nan
    dl[0], de[0] = 0.0, 0.0
    t[1], de[1] = -100, 0.0                                                                  # a place of a prompt
    de[2] = 0.0
    de[3] = 0.0
    _, lse, ent, _, _ = ops.g10_log_probs(x, t, entropy=True)
    g = ops.g10_log_probs_backward(dl, x, t, lse, de, ent)
    assert ent[:3].isnan().all() and not g[:2].any() and g[2].isnan().all()
    K.check(dict(dlogits=g[3:]), K.log_probs(x[3:], t[3:], 1.0, dlogp=dl[3:], dentropy=de[3:], near=64.0)[0])
    g = ops.g10_log_probs_backward(None, x, None, lse, de, ent)
    assert not g[:4].any()
    leaf = x.clone().requires_grad_()
    logp, ent = ops.log_probs(leaf, t, entropy=True)
    logp[1:2].sum().backward()                                                               # a loss of one row, whose token does not count
    assert not leaf.grad.any()


@pytest.mark.parametrize("vocab", [60, 3001, 70000])
@pytest.mark.parametrize("dtype", TYPES)
def test_tokens_outside_the_row_that_have_no_share(ops, dtype, vocab):
    """Such a token's logp is NaN, and so is its row's gradient, but not where logp has no share in the loss."""
    x, t, dl, de = make(6, vocab, dtype)
    t[0], t[1], t[2], t[3] = vocab, -1, 2 ** 40, -(2 ** 40)
    dl[0], de[0], dl[1], dl[4] = 0.0, 0.0, 0.0, 0.0                                          # no share at all; none of logp; (the last: nor a token outside)
    _, lse, ent, _, _ = ops.g10_log_probs(x, t, entropy=True)
    for d2 in (de, None):
        g = ops.g10_log_probs_backward(dl, x, t, lse, d2, ent)
        assert not g[0].any() and g[2:4].isnan().all()
        K.check(dict(dlogits=g), K.log_probs(x, t, 1.0, dlogp=dl, dentropy=d2, near=64.0)[0])
    with_tokens, without = (ops.g10_log_probs_backward(None, x, t1, lse, de, ent) for t1 in (t, None))
    assert torch.equal(with_tokens, without)                                                 # nothing of logp: the tokens do not matter
    K.check(dict(dlogits=without), K.log_probs(x, None, 1.0, dentropy=de, near=64.0)[0])
    leaf = x.clone().requires_grad_()
    logp, ent = ops.log_probs(leaf, t, entropy=True)
    (ent * de).sum().backward()
    assert torch.equal(leaf.grad, without)
