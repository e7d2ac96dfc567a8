"""The trace of the lean decoder is a well-formed step of the same model."""
import numpy as np

from paper_2310_09443_amd import lean, traces


def test_trace():
    full, w = traces.decoder48().trace, lean.decoder48_lean().trace
    assert (w.dur_ns > 0).all() and (w.size_bytes > 0).all()
    assert w.use_kernel.max() == w.K - 1 and w.use_tensor.max() < w.N
    assert len(np.unique(w.use_tensor)) == w.N                        # every tensor is used
    assert int(w.size_bytes.sum()) < int(full.size_bytes.sum())
