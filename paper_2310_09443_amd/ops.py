"""The operators of a training step that stand next to the planner, on torch tensors (include/g10_ops.h is the C ABI below).

  norm_rope     norms of queries and keys with the rotation by position, one pass over both
  attention     attention with a sliding window and first tokens that stay visible; scores never leave the chip
  AdamW         one update over all weights at once, moments in 32 or 8 bits, and the norm of all gradients
  embed         rows of a table by token
  norm          norms of whole rows, centred or not
  gated         act(x gate) * (x up), the first half of a gated MLP
  log_probs     logarithms of given tokens' probabilities, entropy, the likeliest tokens

All but AdamW are differentiable; the g10_* functions beside them are the forward and backward calls
themselves.  Work is enqueued on the current stream of the tensors' device and not waited for; outputs and workspaces are
torch's, allocated on that stream.  What the library would refuse raises ValueError, before anything is launched.  Rows that no one
stride describes are copied first: `logits[:, :-1]` of [batch, token, vocab] is (shift the tokens instead, or leave the last one out before the
logits are made).  The marshalling is C++ (csrc/g10_torch.cpp): in Python it would take longer than the kernels of a small step.
"""
from __future__ import annotations

import ctypes as C
import math

import torch

from . import binding

EXPORTS = ["g10_norm_rope", "g10_norm_rope_workspace", "g10_norm_rope_backward", "g10_attention_workspace", "g10_attention",
           "g10_attention_backward_workspace", "g10_attention_backward", "g10_adamw_blocks", "g10_adamw_create", "g10_adamw_step",
           "g10_grad_norm", "g10_adamw_free",
           "g10_embed", "g10_embed_backward_workspace", "g10_embed_backward", "g10_norm", "g10_norm_backward_workspace", "g10_norm_backward",
           "g10_log_probs_workspace", "g10_log_probs", "g10_log_probs_backward", "g10_gated_workspace", "g10_gated",
           "g10_gated_backward_workspace", "g10_gated_backward"]
LAYER = EXPORTS.index("g10_embed")               # the operators around attention, from here on

F32, F16, BF16, E4M3 = 0, 1, 2, 3
SILU, GELU = 0, 1
LOG_PROBS_TOP = 64
ADAMW_BLOCK = 256
_TYPE = {torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16}
_PTR, _I64, _U32, _U64 = C.c_void_p, C.c_int64, C.c_uint32, C.c_uint64


# The structs of the C ABI, for callers that make its calls themselves.
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


class _Embed(C.Structure):
    _fields_ = [(n, _PTR) for n in ("ids", "table", "out", "dout", "dtable")] + \
               [(n + "_stride", _I64) for n in ("table", "out", "dout", "dtable")] + \
               [(n, _U32) for n in ("tokens", "vocab", "dim")] + [("scale", C.c_float), ("type", _U32), ("ids_64", _U32)]


class _Norm(C.Structure):
    _fields_ = [(n, _PTR) for n in ("x", "dy", "weight", "bias", "out", "dweight", "dbias")] + \
               [(n + "_stride", _I64) for n in ("x", "dy", "out")] + \
               [("rows", _U32), ("dim", _U32), ("eps", C.c_float), ("center", _U32), ("type", _U32), ("weight_type", _U32)]


class _LogProbs(C.Structure):
    _fields_ = [(n, _PTR) for n in ("logits", "tokens", "logp", "lse", "entropy", "top_logp", "top_ids", "dlogp", "dentropy", "dlogits")] + \
               [("logits_stride", _I64), ("dlogits_stride", _I64), ("rows", _U32), ("vocab", _U32), ("top", _U32), ("scale", C.c_float),
                ("ignore", _I64), ("type", _U32)]


class _Gated(C.Structure):
    _fields_ = [(n, _PTR) for n in ("x", "gate", "up", "h", "dh", "dx", "dgate", "dup")] + \
               [(n + "_stride", _I64) for n in ("x", "gate", "up", "h", "dh", "dx", "dw")] + \
               [(n, _U32) for n in ("tokens", "dim", "inner", "act", "out_in", "type")]


_ready = _torch = None


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
        for n, args, room in (("g10_embed", _Embed, False), ("g10_embed_backward", _Embed, True), ("g10_norm", _Norm, False), ("g10_norm_backward", _Norm, True),
                              ("g10_log_probs", _LogProbs, True), ("g10_log_probs_backward", _LogProbs, False), ("g10_gated", _Gated, True),
                              ("g10_gated_backward", _Gated, True)):
            getattr(lib, n).argtypes = [C.POINTER(args)] + ([_PTR, _U64] if room else []) + [_PTR]
            if room:
                getattr(lib, n + "_workspace").argtypes = [C.POINTER(args), ws]
        _ready = lib
    return _ready


def _calls():
    """The marshalling module (csrc/g10_torch.cpp), bound to the loaded library."""
    global _torch
    if _torch is None:
        lib = _load()
        try:
            from . import _g10_torch
        except ImportError as e:
            raise ImportError("paper_2310_09443_amd/_g10_torch.so is missing: run `python -m paper_2310_09443_amd.build`") from e
        at = [C.cast(getattr(lib, n), _PTR).value for n in EXPORTS]
        _g10_torch.bind([x for n, x in zip(EXPORTS[:LAYER], at) if n != "g10_adamw_blocks"])
        _g10_torch.bind_layer(at[LAYER:])
        _torch = _g10_torch
    return _torch


def _need(ok, what):
    if not ok:
        raise ValueError(what)


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


def g10_norm_rope(q, k, table, positions, q_weight=None, k_weight=None, eps=1e-6, interleaved=False):
    """Queries and keys ([batch, token, head, dim] or [token, head, dim], either may be None), each head's values divided by the
    root of their mean square and multiplied by the weight, their first table.shape[1] values turned by the position's angles.
    `interleaved`: pairs are neighbours, else (i, i + rot/2).  A position outside the table gives NaN.  Returns (q, k)."""
    return _calls().norm_rope(q, k, table, positions, q_weight, k_weight, eps, interleaved, False, None, None)


def g10_norm_rope_backward(dq, dk, q, k, table, positions, q_weight=None, k_weight=None, eps=1e-6, interleaved=False):
    """Gradients of g10_norm_rope's inputs from those of its outputs: (dq, dk, dq_weight, dk_weight), None where there is none."""
    return _calls().norm_rope(q, k, table, positions, q_weight, k_weight, eps, interleaved, True, dq, dk)


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
def g10_attention(q, k, v, causal=True, window=0, sinks=0, scale=None, q_start=None, k_start=None, k_len=None, max_q=None, max_k=None):
    """softmax(scale q k^T) v over the keys each query sees, which stand side by side: q [batch, token, head, dim], k and v
    [batch, token, kv_head, dim], with `k_len` (int32 [batch]) keys in use; or packed: [token, head, dim] with `q_start` and
    `k_start` (int32 [batch + 1], not falling), `max_q` and `max_k` the longest sequences' lengths (they steer how the work is cut).
    The last query of a sequence stands at its last key.  causal: no key behind the query; window w > 0: only the last w keys up
    to the query's own (not causal: fewer than w places away), and the first `sinks` ones.  Returns (o, lse); a query that sees no key has
    o = 0 and lse = -inf, as do rows of packed tensors that belong to no sequence (padding before the first or behind the last one)."""
    return _calls().attention(q, k, v, causal, window or 0, sinks, scale, q_start, k_start, k_len, max_q, max_k)


def g10_attention_backward(do, q, k, v, o, lse, causal=True, window=0, sinks=0, scale=None, q_start=None, k_start=None, k_len=None,
                           max_q=None, max_k=None):
    """Gradients (dq, dk, dv) from that of o, with g10_attention's inputs and outputs.  Keys past k_len and rows that belong to no sequence
    get zeros."""
    return _calls().attention_backward(do, q, k, v, o, lse, causal, window or 0, sinks, scale, q_start, k_start, k_len, max_q, max_k)


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


# ----------------------------------------------------------------------------------------------------------- embeddings
def g10_embed(ids, table, scale=1.0):
    """scale * table[ids]: ids of any shape (int32 or int64), table [rows, dim]; [*ids.shape, dim].  An id outside the table gives NaN."""
    return _calls().embed(ids, table, scale)


def g10_embed_backward(dout, ids, rows, scale=1.0):
    """The table's gradient, [rows, dim], from that of g10_embed's output: each row the sum over its tokens, in the same order every time, zeros
    where there are none.  Ids outside the table have no part in it."""
    return _calls().embed_backward(dout, ids, rows, scale)


class _EmbedFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, table, ids, scale):
        ctx.save_for_backward(ids)
        ctx.args = table.shape[0], scale
        return g10_embed(ids, table, scale)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dout):
        return g10_embed_backward(dout, ctx.saved_tensors[0], *ctx.args), None, None


def embed(ids, table, scale=1.0):
    """g10_embed, differentiable in the table.  What is kept for the backward pass: the ids."""
    return _EmbedFn.apply(table, ids, float(scale))


# -------------------------------------------------------------------------------------------------------- norms of rows
def g10_norm(x, weight=None, bias=None, eps=1e-6, center=False):
    """Rows of x ([..., dim]), less their mean with `center` (layer norm), divided by the root of the mean square of what is left, times the
    weight, plus the bias ([dim], either may be None; of x's type or both float32)."""
    return _calls().norm(x, weight, bias, eps, center, False, None)[0]


def g10_norm_backward(dy, x, weight=None, bias=None, eps=1e-6, center=False):
    """Gradients of g10_norm's inputs from that of its output: (dx, dweight, dbias), None where there is none."""
    return _calls().norm(x, weight, bias, eps, center, True, dy)


class _NormFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps, center):
        ctx.save_for_backward(x, weight, bias)
        ctx.args = eps, center
        return g10_norm(x, weight, bias, eps, center)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        return (*g10_norm_backward(dy, *ctx.saved_tensors, *ctx.args), None, None)


def norm(x, weight=None, bias=None, eps=1e-6, center=False):
    """g10_norm, differentiable in x, weight and bias.  The backward pass works the statistics out again from x: nothing else is kept."""
    return _NormFn.apply(x, weight, bias, float(eps), bool(center))


# ----------------------------------------------------------------------------------------------------------- gated MLP
def g10_gated(x, gate, up, act="silu"):
    """act(x gate) * (x up): x [..., dim], gate and up [dim, inner], in float16 or bfloat16; act "silu" or "gelu" (with the error
    function).  Weights kept as [inner, dim] are given transposed (`w.t()`) and read where they lie.  Sums in 32 bits, one rounding."""
    return _calls().gated(x, gate, up, act)


def g10_gated_backward(dh, x, gate, up, act="silu"):
    """Gradients (dx, dgate, dup) from that of g10_gated's output; the weights' lie as the weights do.  Both products of the forward pass are
    made again.  Needs room for the gradients of both products, in x's type: in float16 one of them above 65504 is infinite from there on, and one below
    6e-5 has fewer bits.  All three gradients are made, whichever of the inputs need one."""
    return _calls().gated_backward(dh, x, gate, up, act)


class _GatedFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, gate, up, act):
        ctx.save_for_backward(x, gate, up)
        ctx.act = act
        return g10_gated(x, gate, up, act)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dh):
        return (*g10_gated_backward(dh, *ctx.saved_tensors, ctx.act), None)


def gated(x, gate, up, act="silu"):
    """g10_gated, differentiable in x and both weights.  What is kept for the backward pass: x and the weights."""
    return _GatedFn.apply(x, gate, up, act)


# ---------------------------------------------------------------------------------------------------- log probabilities
def g10_log_probs(logits, tokens=None, entropy=False, top=0, scale=1.0, ignore=-100):
    """Of softmax(scale * logits) over the last dimension: (logp, lse, entropy, top_logp, top_ids), float32 and ids int64, None where not asked for.
    logp: the logarithm of the given tokens' probabilities (`tokens` [...], int64 or int32; 0 for a token equal to `ignore`, NaN for another one outside the
    vocabulary); lse: the logarithm of the sum of exponentials (rounded where it lies: of a row of -1e9 it is -1e9, while logp goes by distances from the
    largest logit); entropy: in nats; top: that many likeliest tokens (up to 64), [..., top], equal
    ones in their own order.  Places of -inf have no probability; a row of nothing else has lse = logp = -inf and entropy 0."""
    return _calls().log_probs(logits, tokens, entropy, top, scale, ignore)


def g10_log_probs_backward(dlogp, logits, tokens, lse, dentropy=None, entropy=None, scale=1.0, ignore=-100):
    """The logits' gradient from those of logp and entropy (either may be None), with g10_log_probs's lse and entropy.  Rows whose lse is 64 or more, of
    16-bit logits 256, either side of zero, are summed again: their lse is rounded too much to take probabilities from."""
    return _calls().log_probs_backward(dlogp, logits, tokens, lse, dentropy, entropy, scale, ignore)


class _LogProbsFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, tokens, entropy, scale, ignore):
        logp, lse, ent, _, _ = g10_log_probs(logits, tokens, entropy, 0, scale, ignore)
        ctx.save_for_backward(logits, tokens, lse, ent)
        ctx.args = scale, ignore
        return (logp, ent) if entropy else logp

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dlogp, dentropy=None):
        logits, tokens, lse, ent = ctx.saved_tensors
        return (g10_log_probs_backward(dlogp, logits, tokens, lse, dentropy, ent, *ctx.args), None, None, None, None)


def log_probs(logits, tokens, entropy=False, scale=1.0, ignore=-100):
    """g10_log_probs's logp, or (logp, entropy), differentiable in the logits.  What is kept for the backward pass: the logits and a number or two a
    row; a loss is `-log_probs(logits, tokens).sum() / n`."""
    _need(tokens is not None or entropy, "tokens or entropy is needed")
    return _LogProbsFn.apply(logits, tokens, bool(entropy), float(scale), int(ignore))


# ---------------------------------------------------------------------------------------------------------------- AdamW
class AdamW:
    """AdamW over all of `params` (contiguous tensors of one type that share no memory: float32, float16 or bfloat16) in one launch a step.

    state_bits 32: moments `m` and `v` in float32.  8: `m` and the root of v in float8_e4m3fn, in blocks of 256 values with a float32
    scale each (`m_scale`, `v_scale`): a quarter of the memory.  They are flat tensors, every parameter's part beginning at a multiple
    of 256 (`starts`); saving and loading them and `steps` is all a checkpoint needs.  8-bit moments are rounded to nearest in the first 16 steps
    and then so that their mean over steps is right (to nearest, small changes would be lost in every step).  `copies`: tensors of float16 or bfloat16, one for each
    parameter or None, that receive the updated values in the same pass.  The parameters' memory stays in place until close(); a step that finds it
    elsewhere raises ValueError.  The first step or norm makes the library's tables and cannot be captured into a graph, later ones can.  Steps and norms of one object share a workspace: they must not overlap on two streams."""

    def __init__(self, params, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, state_bits=32, copies=None):
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
        written = [(t, f"{n}[{i}]") for n, ts in (("params", params), ("copies", copies)) for i, t in enumerate(ts) if t is not None and t.numel()]
        spans = sorted((t.data_ptr(), t.data_ptr() + t.numel() * t.element_size(), n) for t, n in written)
        for (_, end, a), (begin, _, b) in zip(spans, spans[1:]):        # two updates of one place at once: either may win
            _need(end <= begin, f"{a} and {b} share memory")
        self.params, self.copies, self.device = params, copies, dev
        self.lr, self.betas, self.eps, self.weight_decay, self.state_bits = lr, betas, eps, weight_decay, state_bits
        self.steps = 0
        self.starts, at = [], 0
        for p in params:
            self.starts.append(at)
            at += -(-p.numel() // ADAMW_BLOCK) * ADAMW_BLOCK
        st = torch.float32 if state_bits == 32 else torch.float8_e4m3fn
        m, v = (torch.zeros(at, dtype=torch.float32 if state_bits == 32 else torch.uint8, device=dev).view(st) for _ in range(2))
        scales = [torch.zeros(at // ADAMW_BLOCK, device=dev) for _ in range(2)] if state_bits == 8 else [None, None]
        self._state = m, v, *scales
        self._core = _calls().AdamwCore(params, copies, *self._state)

    # What the steps work on: copied into (`opt.m.copy_(saved)`), not replaced.
    m = property(lambda self: self._state[0])
    v = property(lambda self: self._state[1])
    m_scale = property(lambda self: self._state[2])
    v_scale = property(lambda self: self._state[3])

    def grad_norm(self, grads=None, max_norm=float("inf")):
        """The norm of all gradients together, summed in 64 bits: a tensor of one number on the device."""
        return self._core.grad_norm(grads, max_norm)

    def step(self, grads=None, max_norm=None, coefficient=None):
        """One update; `grads`: one for each parameter (default: its .grad), None leaves a parameter and its moments as they are.
        max_norm: the gradients are scaled so that their norm together is at most this; returns the norm before (a device tensor, no
        waiting), and a norm that is not finite leaves parameters and moments as they are.  coefficient: a float32 device tensor of one number
        that multiplies the gradients instead (not finite: the same).

        `steps`, whose number the bias corrections go by, counts the calls with a gradient for any parameter.  It is one number for all: a parameter whose first
        gradient comes late is corrected as if the ones before had been 0.  Whether a norm was finite is known on the device only, so such a call counts too; a
        program that looks at the norm may take it back (`opt.steps -= 1`)."""
        some, norm = self._core.step(grads, self.lr, self.betas[0], self.betas[1], self.eps, self.weight_decay, self.steps + 1, max_norm, coefficient)
        self.steps += some
        return norm

    def close(self):
        """Gives the library's tables of the parameters back, after waiting for the device."""
        if getattr(self, "_core", None) is not None:
            self._core.close()
