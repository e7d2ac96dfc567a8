"""What only the library refuses is a ValueError as well."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    from paper_2310_09443_amd import ops
    return ops


def test_more_heads_than_a_grid_holds(ops):
    q = torch.zeros(1, 1, 64, 8, dtype=torch.float16, device="cuda").expand(1 << 18, 1, 64, 8)
    with pytest.raises(ValueError, match="g10_attention"):
        ops.g10_attention(q, q, q)


def test_more_heads_than_a_rotation_takes(ops):
    q = torch.zeros(1, 1, 70000, 8, dtype=torch.float16, device="cuda")
    table, pos = torch.zeros(1, 8, device="cuda"), torch.zeros(1, 1, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError, match="g10_norm_rope"):
        ops.g10_norm_rope(q, None, table, pos)
    with pytest.raises(ValueError, match="g10_norm_rope"):
        ops.g10_norm_rope_backward(q, None, q, None, table, pos)


def test_numbers_of_an_update(ops):
    p, g = [torch.ones(10, device="cuda")], [torch.ones(10, device="cuda")]
    for change in (dict(lr=math.nan), dict(lr=math.inf), dict(weight_decay=math.nan), dict(betas=(1.0, 0.9)), dict(betas=(0.9, -0.1)), dict(eps=-1.0), dict(eps=math.inf)):
        opt = ops.AdamW(p)
        for name, x in change.items():
            setattr(opt, name, x)
        with pytest.raises(ValueError, match="g10_adamw_step"):
            opt.step(g)
        assert opt.steps == 0 and (p[0] == 1).all()
        opt.close()
