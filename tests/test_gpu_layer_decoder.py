"""The small decoder's ids and targets: what does not count in the loss, ids from the table's end, and the ones outside it."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def model():
    from paper_2310_09443_amd import lean
    m = lean.Decoder(vocab=120, dim=64, layers=1, heads=2, kv_heads=1, inner=96, max_len=64)
    yield m
    m.close()


def ids(seed=0):
    return torch.randint(0, 120, (3, 20), generator=torch.Generator().manual_seed(seed)).cuda()


def wanted(model, x, t):
    """The mean over the targets that count by torch, and the output weight's gradient."""
    loss = torch.nn.functional.cross_entropy(model.logits(x).float().flatten(0, 1), t.flatten())
    (grad,) = torch.autograd.grad(loss, model.layers[0]["head"])
    return float(loss.detach()), grad.double()


@pytest.mark.parametrize("ends", [2, 3])
def test_the_loss_is_the_mean_over_the_targets_that_count(model, ends):
    """Off by the additions of some 60 terms in 32 bits, on either side, and of each term's own few roundings: 2^-24 (2 60 + 40); the gradient by the logits'
    gradient's rounding to 16 bits and its own, on either side."""
    x = ids(ends)
    x[:ends, -1] = -100                                                                      # texts that end one token earlier
    loss, grad = wanted(model, x[:, :-1], x[:, 1:])
    got, norm = model.step(x)
    assert abs(float(got) - loss) <= 2 ** -24 * 160 * loss and float(norm) > 0
    assert float((model.layers[0]["head"].grad.double() - grad).norm()) <= 4 * 2 ** -8 * float(grad.norm())
