"""Scales of the log probabilities that 32 bits do not hold in powers of two, in which the exponentials are taken: a logit of 0 would come out as 0 times
infinity.  Refused before anything reaches a device."""
import ctypes as C

import pytest

from paper_2310_09443_amd import binding, ops
from test_layer_abi import call, log_probs_args


@pytest.mark.parametrize("scale", [2.1e38, 2.4e38, 3.4e38, 0.0, -1.0, 1e-46])
def test_scales_beyond_the_range_are_refused(scale):
    for name in ("g10_log_probs", "g10_log_probs_backward"):
        assert call(ops._load(), name, C.byref(log_probs_args(scale=scale))) == binding.EINVAL


@pytest.mark.parametrize("scale", [2e38, 1.0, 1e-38])
def test_scales_within_are_taken(scale):
    n = C.c_uint64()
    assert ops._load().g10_log_probs_workspace(C.byref(log_probs_args(scale=scale)), C.byref(n)) == 0
