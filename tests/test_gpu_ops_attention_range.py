"""Rows that one key nearly takes whole, with a value of next to nothing: what comes out is the sum over thousands of keys whose probabilities lie
far below the largest."""
import math

import pytest
import torch

import opscheck as O

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    from paper_2310_09443_amd import ops
    return ops


# queries and heads that take the kernel for many queries, and the one for few (whole blocks, shares)
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("gap", [0, 6, 12, 15, 17, 18])
@pytest.mark.parametrize("nq, heads, dim, nk", [(640, 16, 64, 4096), (640, 16, 128, 32768), (1, 2, 128, 700), (1, 2, 64, 4096), (3, 2, 128, 32768)])
def test_a_key_that_takes_nearly_all(ops, nq, heads, dim, nk, gap, dtype):
    g = torch.Generator().manual_seed(nk + gap)
    scale = 0.25
    q, k = torch.zeros(1, nq, heads, dim, dtype=dtype), torch.zeros(1, nk, heads, dim, dtype=dtype)
    q[..., 0], k[0, 0, :, 0] = 4.0, gap                               # scores: `gap` for one key, 0 for the others
    k[0, 1:, :, 1:] = torch.randn(nk - 1, heads, dim - 1, generator=g).to(dtype)
    v = (torch.randn(1, nk, heads, dim, generator=g) * 0.25 + 1).to(dtype)
    v[0, 0] = 0
    o, lse = ops.g10_attention(q.cuda(), k.cuda(), v.cuda(), causal=False, scale=scale)
    p = math.exp(-gap) / (1 + (nk - 1) * math.exp(-gap))
    want, A = O.d(v).sum(1, keepdim=True) * p, O.d(v).abs().sum(1, keepdim=True) * p
    # scores are exact; an exponential is good to 4 u of 32 bits and the rounding of its argument; one rounding of each P, one of o, sums of nk terms
    off = O.u(dtype) + (8 + 2 * nk + 4 * gap) * O.U32
    O.assert_near(o, want.expand(o.shape), (O.rounding(want, dtype) + off * A).expand(o.shape), "o")
    want = torch.full(lse.shape, gap + math.log1p((nk - 1) * math.exp(-gap)), dtype=O.F64)
    O.assert_near(lse, want, (8 + nk + 8 * gap) * O.U32 + 8 * O.U32 * (1 + want), "lse")
