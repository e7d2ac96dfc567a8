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


def test_what_counts_as_a_step(ops):
    """A call without any gradient changes nothing, the number that the bias corrections go by either."""
    g = [torch.randn(300, device="cuda"), torch.randn(7, 5, device="cuda")]
    a, b = ([torch.ones_like(x) for x in g] for _ in range(2))
    oa, ob = ops.AdamW(a), ops.AdamW(b)
    for k in range(3):
        for _ in range(k):
            assert oa.step([None, None]) is None and oa.step([None, None], coefficient=torch.ones(1, device="cuda")) is None
            assert float(oa.step([None, None], max_norm=1.0)) == 0.0
            assert oa.step() is None                                  # no parameter has a .grad
        oa.step(g)
        ob.step(g)
        assert oa.steps == ob.steps == k + 1
    oa.step([None, g[1]])
    assert oa.steps == 4
    ob.step([None, g[1]])
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    oa.close()
    ob.close()


@pytest.mark.parametrize("bits", [8, 32])
def test_tensors_that_are_replaced_are_refused(ops, bits):
    """The library's tables point to the memory of the first step: what is put in its place would be ignored, or worse."""
    def make():
        w = [torch.randn(300, device="cuda"), torch.randn(4, device="cuda"), torch.empty(0, device="cuda")]
        half = [w[0].half(), None, None]
        opt = ops.AdamW(w, state_bits=bits, copies=half)
        opt.step([torch.ones_like(x) for x in w])
        return w, half, opt

    for change in (lambda w, half, opt: setattr(w[1], "data", w[1].data.clone()), lambda w, half, opt: setattr(half[0], "data", half[0].data.clone()),
                   lambda w, half, opt: opt.m.set_(opt.m.clone())):
        w, half, opt = make()
        change(w, half, opt)
        kept, grads = [x.clone() for x in w], [torch.ones_like(x) for x in w]
        for call in (lambda: opt.step(grads), lambda: opt.step(grads, max_norm=1.0), lambda: opt.grad_norm(grads)):
            with pytest.raises(ValueError, match="has moved"):
                call()
        assert opt.steps == 1 and all(torch.equal(x, y) for x, y in zip(w, kept))
        opt.close()
        opt.step(grads)                                                # after close() the tables are made anew, of what is there
        assert opt.steps == 2 and not torch.equal(w[1], kept[1])
        opt.close()
    w, half, opt = make()
    for name in ("m", "v", "m_scale", "v_scale"):
        with pytest.raises(AttributeError):
            setattr(opt, name, torch.zeros(5))
    opt.close()


def test_the_first_step_is_not_captured(ops):
    """It makes the library's tables.  Refused before anything is recorded: what else was captured is whole."""
    w, g, x = torch.ones(300, device="cuda"), torch.ones(300, device="cuda"), torch.zeros(300, device="cuda")
    opt = ops.AdamW([w])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        x.add_(1)
        with pytest.raises(ValueError, match="before the capture"):
            opt.step([g])
        with pytest.raises(ValueError, match="before the capture"):
            opt.grad_norm([g])
    for n in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert (x == n + 1).all() and (w == 1).all() and opt.steps == 0
    opt.step([g])
    with torch.cuda.graph(torch.cuda.CUDAGraph()):
        opt.step([g])
    opt.close()


def test_tensors_that_share_memory_are_refused(ops):
    """They are updated at the same time: which of two updates stays would change from run to run."""
    w = torch.ones(1000, device="cuda")
    h = w.bfloat16()
    for params, copies in (([w, w], None), ([w, w[500:]], None), ([w[:600], w[599:]], None), ([w[:8], w[100:]], [h[:8], h[7:907]]),
                           ([h, w.bfloat16()], [h, None]), ([w.new_ones(4).bfloat16(), h], [h[:4], None])):
        with pytest.raises(ValueError, match="share memory"):
            ops.AdamW(params, copies=copies)
    opt = ops.AdamW([w[:500], w[500:], w[500:500]], copies=[h[:500], h[500:], None])       # side by side is fine
    opt.step([torch.ones(500, device="cuda"), torch.ones(500, device="cuda"), None])
    assert (w < 1).all()
    opt.close()


def test_views_of_one_buffer_move_its_version(ops):
    """A buffer and its views have one version: it moves in every step that writes any of them, and other buffers' do not."""
    flat, other = torch.ones(1000, device="cuda"), torch.ones(50, device="cuda")
    half = torch.ones(1000, dtype=torch.bfloat16, device="cuda")
    opt = ops.AdamW([flat[:300], other, flat[300:]], copies=[half[:300], None, half[300:]])
    one = lambda t: torch.ones(t, device="cuda")                                          # noqa: E731
    for grads, moved in (([one(300), one(50), one(700)], (1, 1, 1)), ([None, None, one(700)], (1, 0, 1)), ([None, one(50), None], (0, 1, 0)),
                         ([one(300), None, one(700)], (1, 0, 1))):
        before = flat._version, other._version, half._version
        opt.step(grads)
        for b, a, m in zip(before, (flat._version, other._version, half._version), moved):
            assert (a > b) == bool(m)
    opt.close()
