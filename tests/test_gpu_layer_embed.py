"""Rows of a table by token and the table's gradient, against the 64-bit formulas."""
import pytest
import torch

import layercheck as L

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    from paper_2310_09443_amd import ops
    return ops


def check(ops, ids, table, dout, scale=1.0):
    got = ops.g10_embed(ids, table, scale)
    assert got.shape == (*ids.shape, table.shape[1]) and got.dtype == table.dtype
    L.assert_near(got, *L.embed(ids, table, scale), "out")
    back = ops.g10_embed_backward(dout, ids, table.shape[0], scale)
    L.assert_near(back, *L.embed_backward(dout, ids, table.shape[0], scale), "dtable")
    assert torch.equal(back, ops.g10_embed_backward(dout, ids, table.shape[0], scale))       # the same bits again


def make(tokens, vocab, dim, dtype, seed=0, ids64=False, frequent=True):
    g = torch.Generator().manual_seed(seed)
    u = torch.rand(tokens, generator=g, dtype=torch.float64)
    ids = ((vocab + 1) ** u).long().clamp(1, vocab) - 1 if frequent else (u * vocab).long()
    r = lambda *s: torch.randn(*s, generator=g).to(dtype).cuda()                             # noqa: E731
    return ids.to(torch.int64 if ids64 else torch.int32).cuda(), r(vocab, dim), r(tokens, dim)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("tokens, vocab, dim", [(1, 1, 1), (1, 7, 8), (3, 5, 64), (63, 10, 24), (64, 10, 512), (65, 100, 520), (200, 1, 40), (1000, 30, 7), (700, 5000, 130),
                                                (4097, 511, 256), (130, 512, 1032), (5, 70000, 16)])
def test_sizes(ops, tokens, vocab, dim, dtype):
    ids, table, dout = make(tokens, vocab, dim, dtype, seed=tokens + dim)
    check(ops, ids, table, dout, scale=0.37)


def test_many_tokens_of_many_rows(ops):
    """More than one tile of the sort and three of its passes; runs over the ends of many pieces beside rows of one token."""
    ids, table, dout = make(20000, 300001, 16, torch.float32, ids64=True)
    check(ops, ids, table, dout)
    ids, table, dout = make(9000, 3000, 96, torch.bfloat16, frequent=False, seed=3)
    ids[1000:6000] = 17                                                                     # one token for most of the batch
    check(ops, ids, table, dout, scale=-2.0)
    ids[:] = 2999
    check(ops, ids, table, dout)


@pytest.mark.parametrize("ids64", [False, True])
def test_ids_outside_the_table(ops, ids64):
    ids, table, dout = make(300, 40, 48, torch.bfloat16, ids64=ids64)
    ids[::7] = -1
    ids[5], ids[6], ids[100] = 40, 2 ** 31 - 1, -2 ** 31
    if ids64:
        ids[101] = 2 ** 32 + 3                                                              # (a row's number in its lower half)
    check(ops, ids, table, dout)
    ids[:] = -5
    check(ops, ids, table, dout)


def test_layouts(ops):
    ids, table, dout = make(60, 33, 64, torch.float16)
    ids3 = ids.view(3, 4, 5).transpose(0, 1)
    check(ops, ids3, table, dout.view(4, 3, 5, 64))
    wide = torch.randn(33, 200, device="cuda").half()
    check(ops, ids, wide[:, 8:72], dout)                                                    # rows of a wider table
    check(ops, ids, wide[:, 3:67], dout)                                                    # not at multiples of 16 bytes
    check(ops, ids, table.t().contiguous().t(), dout.t().contiguous().t())                  # columns contiguous
    check(ops, ids, wide[::2, :64].contiguous(), torch.randn(60, 128, device="cuda").half()[:, 1::2])
    check(ops, ids, table, dout[:1].expand(60, 64))
    check(ops, ids[0], table, dout[0])                                                      # one token, no dimension


def test_no_tokens(ops):
    e = torch.empty(2, 0, dtype=torch.int64, device="cuda")
    table = torch.randn(9, 24, device="cuda")
    assert ops.g10_embed(e, table).shape == (2, 0, 24)
    back = ops.g10_embed_backward(torch.empty(2, 0, 24, device="cuda"), e, 9)
    assert back.shape == (9, 24) and not back.any()


def test_gradient_through_autograd(ops):
    ids, table, dout = make(50, 20, 32, torch.float32)
    table.requires_grad_()
    (ops.embed(ids, table, 3.0) * dout).sum().backward()
    L.assert_near(table.grad, *L.embed_backward(dout, ids, 20, 3.0), "dtable")


def test_refusals(ops):
    ids, table, dout = make(6, 5, 16, torch.float32)
    for bad, match in ((lambda: ops.g10_embed(ids.float(), table), "int32 or int64"), (lambda: ops.g10_embed(ids, table[0]), "rows, dim"),
                       (lambda: ops.g10_embed(ids.cpu(), table), "GPU memory"), (lambda: ops.g10_embed(ids, table.double()), "not supported"),
                       (lambda: ops.g10_embed(ids, table, float("nan")), "finite"), (lambda: ops.g10_embed(ids, table[:0]), "rows, dim"),
                       (lambda: ops.g10_embed_backward(dout[:5], ids, 5), "row for each"), (lambda: ops.g10_embed_backward(dout, ids, 0), "1 to"),
                       (lambda: ops.g10_embed_backward(torch.zeros(6, 65537, device="cuda"), ids, 5), "65536")):
        with pytest.raises(ValueError, match=match):
            bad()


@pytest.mark.parametrize("tokens", [1, 64, 255, 4096, 4097, 5121, 131072, 131073, 300000])
def test_sorts(ops, tokens):
    """Sorted in one workgroup, in tiles of one round and of several, with ids of one, two and three digits."""
    for vocab in (300, 30000, 300000):
        check(ops, *make(tokens, vocab, 8, torch.float32, seed=vocab, frequent=vocab == 300))


def test_a_run_over_many_pieces(ops):
    """More than 64 pieces of one id, and such a run right behind another one."""
    ids, table, dout = make(20000, 50, 72, torch.bfloat16)
    ids[:] = 7
    ids[::3] = 6
    ids[:200] = 49
    check(ops, ids, table, dout)
