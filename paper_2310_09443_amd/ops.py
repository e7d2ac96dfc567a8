"""The operators of a training step that stand next to the planner: binding over the C ABI of include/g10_ops.h.

  norm_rope     norms of queries and keys with the rotation by position, one pass over both
  attention     attention with a sliding window and first tokens that stay visible; scores never leave the chip
  AdamW         one update over all weights at once, moments in 32 or 8 bits, and the norm of all gradients

`norm_rope` and `attention` are differentiable; the g10_* functions beside them are the forward and backward calls
themselves.  Work is enqueued on the current stream of the tensors' device and not waited for; outputs and workspaces are
torch's, allocated on that stream.  What the library would refuse raises ValueError here, before anything is launched.
"""
from __future__ import annotations

import ctypes as C
import math

import torch

from . import binding

EXPORTS = ["g10_norm_rope", "g10_norm_rope_workspace", "g10_norm_rope_backward", "g10_attention_workspace", "g10_attention",
           "g10_attention_backward_workspace", "g10_attention_backward", "g10_adamw_blocks", "g10_adamw_create", "g10_adamw_step",
           "g10_grad_norm", "g10_adamw_free"]

F32, F16, BF16, E4M3 = 0, 1, 2, 3
ADAMW_BLOCK = 256
_TYPE = {torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16}
_PTR, _I64, _U32, _U64 = C.c_void_p, C.c_int64, C.c_uint32, C.c_uint64


class _RopePart(C.Structure):
    _fields_ = [("x", _PTR), ("weight", _PTR), ("dy", _PTR), ("out", _PTR), ("dweight", _PTR), ("x_stride", _I64 * 3),
                ("dy_stride", _I64 * 3), ("out_stride", _I64 * 3), ("heads", _U32)]


class _Rope(C.Structure):
    _fields_ = [("part", _RopePart * 2), ("batch", _U32), ("seq", _U32), ("dim", _U32), ("rot", _U32), ("table", _PTR),
                ("n_positions", _U32), ("positions", _PTR), ("eps", C.c_float), ("type", _U32), ("weight_type", _U32), ("flags", _U32)]


class _Attention(C.Structure):
    _fields_ = [(n, _PTR) for n in ("q", "k", "v", "o", "lse", "d_o", "dq", "dk", "dv")] + \
               [(n + "_stride", _I64 * 3) for n in ("q", "k", "v", "o", "do", "dq", "dk", "dv")] + \
               [(n, _U32) for n in ("batch", "heads", "kv_heads", "dim", "seq_q", "seq_k")] + \
               [(n, _PTR) for n in ("q_start", "k_start", "k_len")] + \
               [(n, _U32) for n in ("max_q", "max_k", "causal", "window", "sinks")] + [("scale", C.c_float), ("type", _U32)]


class _AdamwTensor(C.Structure):
    _fields_ = [("p", _PTR), ("copy", _PTR), ("n", _U64)]


class _AdamwDesc(C.Structure):
    _fields_ = [("tensors", C.POINTER(_AdamwTensor)), ("count", _U32), ("type", _U32), ("grad_type", _U32), ("copy_type", _U32),
                ("state_type", _U32), ("m", _PTR), ("v", _PTR), ("m_scale", _PTR), ("v_scale", _PTR)]


class _AdamwParams(C.Structure):
    _fields_ = [("lr", C.c_double), ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double), ("weight_decay", C.c_double),
                ("step", _U64), ("coefficient", _PTR)]


_ready = None


def _load():
    global _ready
    if _ready is None:
        lib = binding.load()
        ws = C.POINTER(_U64)
        lib.g10_norm_rope.argtypes = [C.POINTER(_Rope), _PTR]
        lib.g10_norm_rope_workspace.argtypes = [C.POINTER(_Rope), ws]
        lib.g10_norm_rope_backward.argtypes = [C.POINTER(_Rope), _PTR, _U64, _PTR]
        for n in ("g10_attention", "g10_attention_backward"):
            getattr(lib, n).argtypes = [C.POINTER(_Attention), _PTR, _U64, _PTR]
            getattr(lib, n + "_workspace").argtypes = [C.POINTER(_Attention), ws]
        lib.g10_adamw_blocks.argtypes = [C.POINTER(_AdamwTensor), _U32, ws]
        lib.g10_adamw_create.argtypes = [C.POINTER(_AdamwDesc), _PTR, C.POINTER(_PTR)]
        lib.g10_adamw_step.argtypes = [_PTR, C.POINTER(_PTR), C.POINTER(_AdamwParams), _PTR]
        lib.g10_grad_norm.argtypes = [_PTR, C.POINTER(_PTR), C.c_float, _PTR, _PTR]
        lib.g10_adamw_free.argtypes = [_PTR]
        lib.g10_adamw_free.restype = None
        _ready = lib
    return _ready


def _need(ok, what):
    if not ok:
        raise ValueError(what)


def _check(rc, what):
    if rc:
        raise binding.G10Error(rc, what)


def _stream(dev):
    return torch.cuda.current_stream(dev).cuda_stream


class _on:
    """The tensors' device for the call, if it is not the current one."""

    def __init__(self, dev):
        self.dev, self.was = dev, None

    def __enter__(self):
        now = torch.cuda.current_device()
        if self.dev.index is not None and now != self.dev.index:
            self.was = now
            torch.cuda.set_device(self.dev)

    def __exit__(self, *_):
        if self.was is not None:
            torch.cuda.set_device(self.was)


def _workspace(fn, args, dev, what):
    n = _U64()
    _check(fn(C.byref(args), C.byref(n)), what)
    return (torch.empty(n.value, dtype=torch.uint8, device=dev) if n.value else None), n.value


def _ptr(t):
    return None if t is None else t.data_ptr()


def _on_device(t, name, dev=None):
    _need(isinstance(t, torch.Tensor), f"{name} must be a tensor")
    _need(t.is_cuda, f"{name} must lie in GPU memory")
    _need(dev is None or t.device == dev, f"{name} must lie on the device of the other tensors")


# ---------------------------------------------------------------------------------------------------- norm and rotation
def rope_table(n_positions, rot, base=10000.0, device="cuda"):
    """[n_positions, rot]: cosines, then sines, of position * base^(-2i / rot).  Angles are worked out in 64 bits: at position
    100 000 a 32-bit angle is off by 0.004."""
    _need(rot % 2 == 0 and rot >= 0, "rot must be even")
    f = float(base) ** (-torch.arange(0, rot, 2, device=device, dtype=torch.float64) / max(rot, 1))
    a = torch.arange(n_positions, device=device, dtype=torch.float64)[:, None] * f
    return torch.cat([a.cos(), a.sin()], 1).to(torch.float32)


def _inner(t):
    """The tensor with its last dimension contiguous."""
    return t if t.shape[-1] <= 1 or t.stride(-1) == 1 else t.contiguous()


def _strides4(t):
    """(batch, token, head) strides of [batch, token, head, dim] or, with batch 1, of [token, head, dim]."""
    s = t.stride()
    return (s[0], s[1], s[2]) if t.dim() == 4 else (0, s[0], s[1])


def _rope_args(q, k, table, positions, q_weight, k_weight, eps, interleaved, grads=None):
    """The struct, the outputs, and what must stay alive until the call is enqueued."""
    _need(q is not None or k is not None, "queries or keys are needed")
    one = q if q is not None else k
    _on_device(one, "q")
    dev, dt = one.device, one.dtype
    _need(dt in _TYPE, f"type {dt} is not supported: float32, float16 or bfloat16")
    _need(one.dim() in (3, 4), "q and k are [batch, token, head, dim] or [token, head, dim]")
    lead, dim = one.shape[:-2], one.shape[-1]
    a = _Rope()
    keep, outs, dws = [], [], []
    wt = None
    for i, (x, w, name) in enumerate(((q, q_weight, "q"), (k, k_weight, "k"))):
        part = a.part[i]
        if x is None:
            _need(w is None, f"{name}_weight without {name}")
            outs.append(None)
            dws.append(None)
            continue
        _on_device(x, name, dev)
        _need(x.dtype == dt and x.shape[:-2] == lead and x.shape[-1] == dim, f"{name} must have the type, tokens and dim of q")
        x = _inner(x)
        out = torch.empty(x.shape, dtype=dt, device=dev)
        part.heads = x.shape[-2]
        part.x, part.out = _ptr(x), _ptr(out)
        part.x_stride[:], part.out_stride[:] = _strides4(x), _strides4(out)
        keep.append(x)
        if w is not None:
            _on_device(w, name + "_weight", dev)
            _need(w.shape == (dim,) and w.dtype in (dt, torch.float32), f"{name}_weight must be [dim], of the inputs' type or float32")
            _need(wt in (None, w.dtype), "both weights must be of one type")
            wt = w.dtype
            w = w.contiguous()
            part.weight = _ptr(w)
            keep.append(w)
        dw = None
        if grads is not None:
            dy = grads[i]
            _on_device(dy, "d" + name, dev)
            _need(dy.shape == x.shape and dy.dtype == dt, f"d{name} must have the shape and type of {name}")
            dy = _inner(dy)
            part.dy = _ptr(dy)
            part.dy_stride[:] = _strides4(dy)
            keep.append(dy)
            if w is not None:
                dw = torch.empty(dim, dtype=w.dtype, device=dev)
                part.dweight = _ptr(dw)
        outs.append(out)
        dws.append(dw)
    _need(0 < dim <= 256, "dim must be 1 to 256")
    _on_device(table, "table", dev)
    _need(table.dtype == torch.float32 and table.dim() == 2 and table.is_contiguous(), "table must be [positions, rot], float32, contiguous")
    rot = table.shape[1]
    _need(rot % 2 == 0 and rot <= dim, "the table's width must be even and at most dim")
    _on_device(positions, "positions", dev)
    _need(positions.dtype in (torch.int32, torch.int64) and positions.shape == lead, "positions must be int32 or int64, one for each token")
    positions = positions.contiguous()
    keep += [table, positions]
    _need(eps >= 0 and math.isfinite(eps), "eps must not be negative")
    a.batch, a.seq = (lead[0], lead[1]) if len(lead) == 2 else (1, lead[0])
    _need(a.batch == 0 or a.seq == 0 or table.shape[0] > 0, "the table has no positions")
    a.dim, a.rot, a.table, a.n_positions, a.positions = dim, rot, _ptr(table), min(table.shape[0], (1 << 32) - 1), _ptr(positions)
    a.eps, a.type, a.weight_type = eps, _TYPE[dt], _TYPE[wt if wt is not None else dt]
    a.flags = (1 if interleaved else 0) | (2 if positions.dtype == torch.int64 else 0)
    return a, outs, dws, keep, dev


def g10_norm_rope(q, k, table, positions, q_weight=None, k_weight=None, eps=1e-6, interleaved=False):
    """Queries and keys ([batch, token, head, dim] or [token, head, dim], either may be None), each head's values divided by the
    root of their mean square and multiplied by the weight, their first table.shape[1] values turned by the position's angles.
    `interleaved`: pairs are neighbours, else (i, i + rot/2).  A position outside the table gives NaN.  Returns (q, k)."""
    a, outs, _, keep, dev = _rope_args(q, k, table, positions, q_weight, k_weight, eps, interleaved)
    with _on(dev):
        _check(_load().g10_norm_rope(C.byref(a), _stream(dev)), "g10_norm_rope")
    return outs[0], outs[1]


def g10_norm_rope_backward(dq, dk, q, k, table, positions, q_weight=None, k_weight=None, eps=1e-6, interleaved=False):
    """Gradients of g10_norm_rope's inputs from those of its outputs: (dq, dk, dq_weight, dk_weight), None where there is none."""
    a, outs, dws, keep, dev = _rope_args(q, k, table, positions, q_weight, k_weight, eps, interleaved, (dq, dk))
    with _on(dev):
        ws, n = _workspace(_load().g10_norm_rope_workspace, a, dev, "g10_norm_rope_workspace")
        _check(_load().g10_norm_rope_backward(C.byref(a), _ptr(ws), n, _stream(dev)), "g10_norm_rope_backward")
    return outs[0], outs[1], dws[0], dws[1]


class _NormRope(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, q_weight, k_weight, table, positions, eps, interleaved):
        ctx.save_for_backward(q, k, q_weight, k_weight, table, positions)
        ctx.args = eps, interleaved
        return g10_norm_rope(q, k, table, positions, q_weight, k_weight, eps, interleaved)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dq, dk):
        q, k, qw, kw, table, positions = ctx.saved_tensors
        return (*g10_norm_rope_backward(dq, dk, q, k, table, positions, qw, kw, *ctx.args), None, None, None, None)


def norm_rope(q, k, table, positions, q_weight=None, k_weight=None, eps=1e-6, interleaved=False):
    """g10_norm_rope, differentiable in q, k and the weights (q and k both given).  The backward pass works the norms out again from
    q and k: nothing else is kept for it."""
    _need(q is not None and k is not None, "q and k are needed")
    return _NormRope.apply(q, k, q_weight, k_weight, table, positions, float(eps), bool(interleaved))


# ------------------------------------------------------------------------------------------------------------ attention
def _rows16(t):
    """The tensor as the kernels read it: rows and heads at multiples of 16 bytes, the last dimension contiguous; copied if it
    is not so already."""
    s = t.stride()
    if (t.numel() == 0 or (s[-1] == 1 and t.data_ptr() % 16 == 0 and all(x % 8 == 0 or n == 1 for x, n in zip(s[:-1], t.shape[:-1]))
                           and 0 <= s[-3] <= 1 << 22)):
        return t
    return t.contiguous() if t.data_ptr() % 16 == 0 and not t.is_contiguous() else t.clone(memory_format=torch.contiguous_format)


def _put(a, name, t):
    # (a dimension of one place is never stepped over: its stride may be anything)
    s = [x if n > 1 else 0 for x, n in zip(t.stride(), t.shape)]
    setattr(a, name, _ptr(t) if t.numel() else None)
    getattr(a, name.replace("d_o", "do") + "_stride")[:] = (s[0], s[1], s[2]) if t.dim() == 4 else (0, s[0], s[1])


def _starts(t, name, dev):
    _on_device(t, name, dev)
    _need(t.dtype == torch.int32 and t.dim() == 1, f"{name} must be a vector of int32")
    return t.contiguous()


def _attention_args(q, k, v, causal, window, sinks, scale, q_start, k_start, k_len, max_q, max_k):
    _on_device(q, "q")
    dev, dt = q.device, q.dtype
    _need(dt in (torch.float16, torch.bfloat16), f"type {dt} is not supported: float16 or bfloat16")
    for t, name in ((k, "k"), (v, "v")):
        _on_device(t, name, dev)
        _need(t.dtype == dt and t.dim() == q.dim(), f"{name} must have the type and dimensions of q")
    packed = q_start is not None or k_start is not None
    _need(q.dim() == (3 if packed else 4), "q, k and v are [batch, token, head, dim], packed sequences [token, head, dim]")
    _need(k.shape == v.shape and k.shape[-1] == q.shape[-1], "k and v must have one shape, and the dim of q")
    heads, kv, dim = q.shape[-2], k.shape[-2], q.shape[-1]
    _need(kv > 0 and heads > 0 and heads % kv == 0, "the heads of q must be a multiple of those of k")
    _need(0 < dim <= 128 and dim % 8 == 0, "dim must be a multiple of 8 up to 128")
    window, sinks = int(window or 0), int(sinks)
    _need(0 <= window < 1 << 30 and 0 <= sinks < 1 << 30, "window and sinks must not be negative")
    scale = dim ** -0.5 if scale is None else float(scale)
    _need(scale > 0 and scale < 3e38, "scale must be above zero")
    a = _Attention()
    keep = []
    if packed:
        _need(q_start is not None and k_start is not None and k_len is None, "packed sequences need q_start and k_start, and no k_len")
        q_start, k_start = _starts(q_start, "q_start", dev), _starts(k_start, "k_start", dev)
        _need(q_start.numel() == k_start.numel() and q_start.numel() > 0, "q_start and k_start must hold a number for each sequence and the end")
        a.q_start, a.k_start, a.batch = _ptr(q_start), _ptr(k_start), q_start.numel() - 1
        a.seq_q, a.seq_k = q.shape[0], k.shape[0]
        a.max_q, a.max_k = (min(max(int(m), 0), n) if m is not None else n for m, n in ((max_q, a.seq_q), (max_k, a.seq_k)))
        keep += [q_start, k_start]
    else:
        _need(k.shape[0] == q.shape[0], "q and k must have one batch")
        a.batch, a.seq_q, a.seq_k = q.shape[0], q.shape[1], k.shape[1]
        if k_len is not None:
            k_len = _starts(k_len, "k_len", dev)
            _need(k_len.numel() == a.batch, "k_len must hold a number for each sequence")
            a.k_len = _ptr(k_len)
            keep.append(k_len)
    _need(max(a.seq_q, a.seq_k) < 1 << 30, "too many tokens")
    a.heads, a.kv_heads, a.dim = heads, kv, dim
    a.causal, a.window, a.sinks, a.scale, a.type = int(bool(causal)), window, sinks, scale, _TYPE[dt]
    q, k, v = _rows16(q), _rows16(k), _rows16(v)
    for name, t in (("q", q), ("k", k), ("v", v)):
        _put(a, name, t)
    return a, (q, k, v), keep, dev, packed


def g10_attention(q, k, v, causal=True, window=0, sinks=0, scale=None, q_start=None, k_start=None, k_len=None, max_q=None, max_k=None):
    """softmax(scale q k^T) v over the keys each query sees, which stand side by side: q [batch, token, head, dim], k and v
    [batch, token, kv_head, dim], with `k_len` (int32 [batch]) keys in use; or packed: [token, head, dim] with `q_start` and
    `k_start` (int32 [batch + 1]), `max_q` and `max_k` the longest sequences' lengths (they steer how the work is cut).
    The last query of a sequence stands at its last key.  causal: no key behind the query; window w > 0: only the last w keys up
    to the query's own (not causal: fewer than w places away), and the first `sinks` ones.  Returns (o, lse); a query that sees no key has
    o = 0 and lse = -inf.  Rows of packed tensors that belong to no sequence are not written."""
    a, (q, k, v), keep, dev, packed = _attention_args(q, k, v, causal, window, sinks, scale, q_start, k_start, k_len, max_q, max_k)
    o = torch.empty(q.shape, dtype=q.dtype, device=dev)
    lse = torch.empty((a.heads, a.seq_q) if packed else (a.batch, a.heads, a.seq_q), dtype=torch.float32, device=dev)
    if not q.numel():
        return o, lse
    _put(a, "o", o)
    a.lse = _ptr(lse)
    with _on(dev):
        ws, n = _workspace(_load().g10_attention_workspace, a, dev, "g10_attention_workspace")
        _check(_load().g10_attention(C.byref(a), _ptr(ws), n, _stream(dev)), "g10_attention")
    return o, lse


def g10_attention_backward(do, q, k, v, o, lse, causal=True, window=0, sinks=0, scale=None, q_start=None, k_start=None, k_len=None,
                           max_q=None, max_k=None):
    """Gradients (dq, dk, dv) from that of o, with g10_attention's inputs and outputs.  Keys past k_len get zeros."""
    a, (q, k, v), keep, dev, packed = _attention_args(q, k, v, causal, window, sinks, scale, q_start, k_start, k_len, max_q, max_k)
    for t, name in ((do, "do"), (o, "o")):
        _on_device(t, name, dev)
        _need(t.shape == q.shape and t.dtype == q.dtype, f"{name} must have the shape and type of q")
    _on_device(lse, "lse", dev)
    _need(lse.dtype == torch.float32 and lse.is_contiguous() and lse.numel() == a.heads * a.seq_q * (1 if packed else a.batch), "lse must be g10_attention's")
    do, o = _rows16(do), _rows16(o)
    dq, dk, dv = (torch.empty(t.shape, dtype=t.dtype, device=dev) for t in (q, k, v))
    if not q.numel() or not a.batch:
        return dq.zero_(), dk.zero_(), dv.zero_()
    for name, t in (("d_o", do), ("o", o), ("dq", dq), ("dk", dk), ("dv", dv)):
        _put(a, name, t)
    a.lse = _ptr(lse)
    with _on(dev):
        ws, n = _workspace(_load().g10_attention_backward_workspace, a, dev, "g10_attention_backward_workspace")
        _check(_load().g10_attention_backward(C.byref(a), _ptr(ws), n, _stream(dev)), "g10_attention_backward")
    return dq, dk, dv


class _AttentionFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, q_start, k_start, k_len, args):
        o, lse = g10_attention(q, k, v, q_start=q_start, k_start=k_start, k_len=k_len, **args)
        ctx.save_for_backward(q, k, v, o, lse, q_start, k_start, k_len)
        ctx.args = args
        return o

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, do):
        q, k, v, o, lse, q_start, k_start, k_len = ctx.saved_tensors
        return (*g10_attention_backward(do, q, k, v, o, lse, q_start=q_start, k_start=k_start, k_len=k_len, **ctx.args), None, None, None, None)


def attention(q, k, v, causal=True, window=0, sinks=0, scale=None, q_start=None, k_start=None, k_len=None, max_q=None, max_k=None):
    """g10_attention's o, differentiable in q, k and v.  What is kept for the backward pass: q, k, v, o and one number a query and head."""
    return _AttentionFn.apply(q, k, v, q_start, k_start, k_len, dict(causal=causal, window=window, sinks=sinks, scale=scale, max_q=max_q, max_k=max_k))


# ---------------------------------------------------------------------------------------------------------------- AdamW
class AdamW:
    """AdamW over all of `params` (contiguous tensors of one type: float32, float16 or bfloat16) in one launch a step.

    state_bits 32: moments `m` and `v` in float32.  8: `m` and the root of v in float8_e4m3fn, in blocks of 256 values with a float32
    scale each (`m_scale`, `v_scale`): a quarter of the memory.  They are flat tensors, every parameter's part beginning at a multiple
    of 256 (`starts`); saving and loading them and `steps` is all a checkpoint needs.  `copies`: tensors of float16 or bfloat16, one for each
    parameter or None, that receive the updated values in the same pass.  The parameters' memory stays in place until close()."""

    def __init__(self, params, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, state_bits=32, copies=None, grad_dtype=None):
        params = list(params)
        _need(len(params) > 0, "no parameters")
        _need(len(params) <= 1 << 20, "too many parameters")
        _need(state_bits in (8, 32), "state_bits must be 8 or 32")
        _need(0 <= betas[0] < 1 and 0 <= betas[1] < 1 and eps >= 0, "betas must be in [0, 1), eps not negative")
        _on_device(params[0], "params[0]")
        dev, dt = params[0].device, params[0].dtype
        _need(dt in _TYPE, f"type {dt} is not supported: float32, float16 or bfloat16")
        for i, p in enumerate(params):
            _on_device(p, f"params[{i}]", dev)
            _need(p.dtype == dt and p.is_contiguous(), f"params[{i}] must be contiguous and of the type of the others")
        copies = list(copies) if copies is not None else [None] * len(params)
        _need(len(copies) == len(params), "copies must be one for each parameter")
        ct = next((c.dtype for c in copies if c is not None), None)
        _need(ct in (None, torch.float16, torch.bfloat16), "copies must be float16 or bfloat16")
        for i, (p, c) in enumerate(zip(params, copies)):
            if c is not None:
                _on_device(c, f"copies[{i}]", dev)
                _need(c.dtype == ct and c.is_contiguous() and c.shape == p.shape, f"copies[{i}] must be contiguous, of one type and its parameter's shape")
        self.params, self.copies, self.device = params, copies, dev
        self.lr, self.betas, self.eps, self.weight_decay, self.state_bits = lr, betas, eps, weight_decay, state_bits
        self.grad_dtype = grad_dtype
        self.steps = 0
        self.starts, at = [], 0
        for p in params:
            self.starts.append(at)
            at += -(-p.numel() // ADAMW_BLOCK) * ADAMW_BLOCK
        st = torch.float32 if state_bits == 32 else torch.float8_e4m3fn
        self.m, self.v = (torch.zeros(at, dtype=torch.float32 if state_bits == 32 else torch.uint8, device=dev).view(st) for _ in range(2))
        self.m_scale = self.v_scale = None
        if state_bits == 8:
            self.m_scale, self.v_scale = (torch.zeros(at // ADAMW_BLOCK, device=dev) for _ in range(2))
        self._h, self._ct = None, ct

    def _handle(self, grad_type):
        if self._h is None:
            n = len(self.params)
            ts = (_AdamwTensor * n)(*((_ptr(p), _ptr(c), p.numel()) for p, c in zip(self.params, self.copies)))
            d = _AdamwDesc(ts, n, _TYPE[self.params[0].dtype], grad_type, _TYPE.get(self._ct, 0), F32 if self.state_bits == 32 else E4M3,
                           _ptr(self.m), _ptr(self.v), _ptr(self.m_scale), _ptr(self.v_scale))
            h = _PTR()
            _check(_load().g10_adamw_create(C.byref(d), _stream(self.device), C.byref(h)), "g10_adamw_create")
            self._h, self._grad_type = h, grad_type
        _need(self._grad_type == grad_type, "the gradients' type changed")
        return self._h

    def _pointers(self, grads):
        """The gradients' addresses, their type, and copies that had to be made."""
        grads = [p.grad for p in self.params] if grads is None else list(grads)
        _need(len(grads) == len(self.params), "grads must be one for each parameter")
        keep, dt, out = [], self.grad_dtype, (_PTR * len(grads))()
        dev, n = self.device, 0
        for i, (g, p) in enumerate(zip(grads, self.params)):
            if g is None:
                continue
            if dt is None:
                dt = g.dtype
                _need(dt in _TYPE, f"gradients of type {dt} are not supported")
            _need(g.device == dev and g.dtype == dt and g.shape == p.shape, f"grads[{i}] must have its parameter's shape and device and the type of the others")
            if not g.is_contiguous():
                g = g.contiguous()
                keep.append(g)
            out[i] = g.data_ptr()
            n += 1
        return out, dt, keep, n

    def grad_norm(self, grads=None, max_norm=float("inf")):
        """The norm of all gradients together, summed in 64 bits: a tensor of one number on the device."""
        _need(max_norm > 0, "max_norm must be above zero")
        out, dt, keep, n = self._pointers(grads)
        if not n:
            return torch.zeros((), device=self.device)
        res = torch.empty(2, device=self.device)
        with _on(self.device):
            _check(_load().g10_grad_norm(self._handle(_TYPE[dt]), out, min(float(max_norm), 3e38), _ptr(res), _stream(self.device)), "g10_grad_norm")
        return res[0]

    def step(self, grads=None, max_norm=None, coefficient=None):
        """One update; `grads`: one for each parameter (default: its .grad), None leaves a parameter and its moments as they are.
        max_norm: the gradients are scaled so that their norm together is at most this; returns the norm before (a device tensor, no
        waiting), and a norm that is not finite leaves everything as it is.  coefficient: a float32 device tensor of one number
        that multiplies the gradients instead (not finite: nothing changes)."""
        _need(max_norm is None or max_norm > 0, "max_norm must be above zero")
        _need(max_norm is None or coefficient is None, "max_norm or coefficient")
        if coefficient is not None:
            _on_device(coefficient, "coefficient", self.device)
            _need(coefficient.dtype == torch.float32 and coefficient.numel() == 1, "coefficient must be one float32 number")
        out, dt, keep, n = self._pointers(grads)
        self.steps += 1
        if not n:
            return None
        lib, s = _load(), None
        with _on(self.device):
            h, s = self._handle(_TYPE[dt]), _stream(self.device)
            p = _AdamwParams(self.lr, self.betas[0], self.betas[1], self.eps, self.weight_decay, self.steps, _ptr(coefficient))
            norm = None
            if max_norm is not None:
                norm = torch.empty(2, device=self.device)
                _check(lib.g10_grad_norm(h, out, min(float(max_norm), 3e38), _ptr(norm), s), "g10_grad_norm")
                p.coefficient = norm.data_ptr() + 4
            _check(lib.g10_adamw_step(h, out, C.byref(p), s), "g10_adamw_step")
        return None if norm is None else norm[0]

    def close(self):
        if getattr(self, "_h", None):
            _load().g10_adamw_free(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
