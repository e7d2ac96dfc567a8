"""The trace of the decoder whose norms and gated MLP keep their inputs alone, and that the one without them is what it was."""
import hashlib

import numpy as np

from paper_2310_09443_amd import lean


def test_trace_with_the_layer_operators():
    a, b = lean.decoder48_lean().trace, lean.decoder48_lean(layer=True).trace
    assert (b.dur_ns > 0).all() and (b.size_bytes > 0).all()
    assert b.use_kernel.max() == b.K - 1 and b.use_tensor.max() < b.N
    assert len(np.unique(b.use_tensor)) == b.N
    assert b.K < a.K and int(b.size_bytes.sum()) < int(a.size_bytes.sum())
    weights = lambda t: sorted(int(x) for x, g in zip(t.size_bytes, t.is_global) if g)[-500:]        # noqa: E731
    assert weights(a) == weights(b)                                                                   # the same model


def test_trace_without_them_is_what_it_was():
    t = lean.decoder48_lean().trace
    data = b"".join(np.ascontiguousarray(x).tobytes() for x in (t.dur_ns, t.size_bytes, t.use_kernel, t.use_tensor))
    assert hashlib.sha256(data).hexdigest()[:12] == "be5f6f61cc38"
