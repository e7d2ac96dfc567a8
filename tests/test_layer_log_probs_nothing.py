"""A differentiable call that nothing is asked of."""
import pytest
import torch

from paper_2310_09443_amd import ops


def test_log_probs_without_tokens_and_entropy_is_refused():
    with pytest.raises(ValueError, match="tokens or entropy"):
        ops.log_probs(torch.zeros(3, 5), None)
