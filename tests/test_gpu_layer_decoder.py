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


def test_ids_outside_the_vocabulary_raise(model):
    """Before anything is launched for them: weights and their gradients stay as they are.  From -vocab on they count from the table's end."""
    x = ids(5)
    before = [t.detach().clone() for w in model.layers for t in w.values()]
    for bad in (120, -121, 2 ** 31 - 1):
        y = x.clone()
        y[1, 3] = bad
        for call in (lambda: model.logits(y), lambda: model.step(y), lambda: model.continue_text(y, 2)):
            with pytest.raises(ValueError, match="ids"):
                call()
    for bad in (-1, 120, -120):                                                              # targets that are no ids, and not -100
        y = x.clone()
        y[2, -1] = bad
        with pytest.raises(ValueError, match="ids|targets"):
            model.step(y)
    assert all(torch.equal(a, t) for a, t in zip(before, (t for w in model.layers for t in w.values())))
    y = x.clone()
    y[y > 100] -= 120
    assert bool((y < 0).any()) and torch.equal(model.logits(y), model.logits(x)) and torch.equal(model.continue_text(y, 2)[:, 20:], model.continue_text(x, 2)[:, 20:])
    assert model.logits(x[:0]).shape == (0, 20, 120)


def test_logits_in_a_graph(model):
    """Nothing is waited for there."""
    x = ids(6)
    with torch.no_grad():
        want = [model.logits(y).clone() for y in (x, x.flip(0))]
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            model.logits(x)
        torch.cuda.current_stream().wait_stream(s)
        g, static = torch.cuda.CUDAGraph(), x.clone()
        with torch.cuda.graph(g):
            out = model.logits(static)
        for y, w in zip((x, x.flip(0), x), (want[0], want[1], want[0])):
            static.copy_(y)
            g.replay()
            assert torch.equal(out, w)
            model.logits(ids(7))
            torch.cuda.synchronize()


def test_logits_of_ids_in_host_memory(model):
    x = ids(8)
    assert torch.equal(model.logits(x.cpu()), model.logits(x))
