"""AdamW as an object of a torch program: what autograd sees of its updates, what counts as a step, tensors that change under it."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    from paper_2310_09443_amd import ops
    return ops


def test_a_graph_made_before_the_update_notices(ops):
    w, still = torch.randn(300, device="cuda", requires_grad=True), torch.randn(300, device="cuda", requires_grad=True)
    half = w.detach().half().requires_grad_()
    opt = ops.AdamW([w.detach(), still.detach()], copies=[half.detach(), None])
    for x in (w, half):
        loss = (x * x).sum()                                          # keeps x for its gradient
        opt.step([torch.ones(300, device="cuda"), None])
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.backward()
        (x * x).sum().backward()                                      # one made after it does not
    loss = (still * still).sum()                                      # without a gradient it was left as it is
    opt.step([torch.ones(300, device="cuda"), None])
    loss.backward()
    opt.close()


def test_tensors_of_inference_mode(ops):
    with torch.inference_mode():
        w = torch.ones(10, device="cuda")
    opt = ops.AdamW([w])
    opt.step([torch.ones(10, device="cuda")])
    assert float(w[0]) < 1
    opt.close()
