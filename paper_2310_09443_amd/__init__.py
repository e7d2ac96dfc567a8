"""G10 tensor-vitality analysis and migration planning on MI355X (HIP, gfx950).

`traces` holds the synthetic workloads; `binding` is the thin ctypes layer over
the C-ABI library built from `csrc/` (it raises if the library is missing).
`ops` holds the operators of a training step that keep less of it (on torch
tensors, same library); `lean` a decoder that uses them, and its trace.
"""
__all__ = ["traces", "binding"]
