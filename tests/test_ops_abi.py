"""The operators' entry points: declared, exported, and what they refuse before anything reaches a device."""
import ctypes as C
import os
import re

import pytest
import torch

from paper_2310_09443_amd import binding, build, ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_header_and_library_have_every_call():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "g10_ops.h")).read(), flags=re.S)
    names = re.findall(r"^\s*(?:int|void)\s+(g10_\w+)\s*\(", text, flags=re.M)
    assert sorted(names) == sorted(ops.EXPORTS)
    if not os.path.exists(build.LIB):
        build.build()
    lib = C.CDLL(build.LIB)
    for n in names:
        assert hasattr(lib, n), n


def test_struct_layouts_match_the_header():
    # (natural alignment of the header's fields)
    assert [C.sizeof(x) for x in (ops._RopePart, ops._Rope, ops._Attention, ops._AdamwTensor, ops._AdamwDesc, ops._AdamwParams)] == \
        [5 * 8 + 9 * 8 + 8, 2 * 120 + 16 + 8 + 8 + 8 + 16, 9 * 8 + 24 * 8 + 24 + 24 + 20 + 8 + 4, 24, 8 + 5 * 4 + 4 + 4 * 8, 5 * 8 + 16]


def test_null_arguments_are_refused():
    lib = ops._load()
    n = C.c_uint64()
    assert lib.g10_norm_rope(None, None) == binding.EINVAL
    assert lib.g10_norm_rope_backward(None, None, 0, None) == binding.EINVAL
    assert lib.g10_norm_rope_workspace(None, C.byref(n)) == binding.EINVAL
    assert lib.g10_attention(None, None, 0, None) == binding.EINVAL
    assert lib.g10_attention_backward(None, None, 0, None) == binding.EINVAL
    assert lib.g10_attention_workspace(C.byref(ops._Attention()), None) == binding.EINVAL
    assert lib.g10_adamw_create(None, None, None) == binding.EINVAL
    assert lib.g10_adamw_step(None, None, None, None) == binding.EINVAL
    assert lib.g10_grad_norm(None, None, 1.0, None, None) == binding.EINVAL
    assert lib.g10_adamw_blocks(None, 1, C.byref(n)) == binding.EINVAL
    lib.g10_adamw_free(None)


def rope_args(**kw):
    a = ops._Rope()
    a.batch, a.seq, a.dim, a.rot, a.n_positions, a.eps, a.type, a.weight_type = 1, 2, 64, 64, 8, 1e-6, ops.BF16, ops.BF16
    a.table = a.positions = 4096
    for p in a.part:
        p.heads, p.x, p.out, p.dy = 2, 4096, 4096, 4096
        for s in (p.x_stride, p.out_stride, p.dy_stride):
            s[:] = 256, 128, 64
    for n, x in kw.items():
        setattr(a, n, x)
    return a


@pytest.mark.parametrize("bad", [dict(dim=0), dict(dim=257), dict(rot=63), dict(rot=66), dict(eps=-1.0), dict(eps=float("nan")), dict(type=3),
                                 dict(weight_type=ops.F16), dict(table=None), dict(positions=None), dict(n_positions=0), dict(flags=4)])
def test_rope_refuses(bad):
    lib, n = ops._load(), C.c_uint64()
    assert lib.g10_norm_rope_workspace(C.byref(rope_args()), C.byref(n)) == 0 and n.value == 0
    assert lib.g10_norm_rope(C.byref(rope_args(**bad)), None) == binding.EINVAL
    assert lib.g10_norm_rope_workspace(C.byref(rope_args(**bad)), C.byref(n)) == binding.EINVAL


def test_rope_refuses_parts():
    lib = ops._load()
    for field, x in (("x", None), ("out", None), ("dy", None), ("x", 4097), ("dweight", 4096)):
        a = rope_args()
        setattr(a.part[1], field, x)
        assert lib.g10_norm_rope_backward(C.byref(a), None, 0, None) == binding.EINVAL, field
    a = rope_args()
    a.part[0].weight = a.part[0].dweight = 4096
    assert lib.g10_norm_rope_backward(C.byref(a), None, 0, None) == binding.EINVAL               # no workspace
    a.part[0].heads, a.part[1].heads = 60000, 6000
    assert lib.g10_norm_rope(C.byref(a), None) == binding.EINVAL


def attention_args(**kw):
    a = ops._Attention()
    a.batch, a.heads, a.kv_heads, a.dim, a.seq_q, a.seq_k, a.scale, a.type = 2, 4, 2, 64, 8, 8, 1.0, ops.BF16
    for n in ("q", "k", "v", "o", "lse", "d_o", "dq", "dk", "dv"):
        setattr(a, n, 4096)
    for n in ("q", "k", "v", "o", "do", "dq", "dk", "dv"):
        getattr(a, n + "_stride")[:] = 2048, 256, 64
    for n, x in kw.items():
        if n.endswith("_stride"):
            getattr(a, n)[:] = x
        else:
            setattr(a, n, x)
    return a


@pytest.mark.parametrize("bad", [dict(dim=0), dict(dim=60), dict(dim=136), dict(heads=3), dict(kv_heads=0), dict(type=ops.F32), dict(scale=0.0),
                                 dict(scale=float("nan")), dict(scale=float("inf")), dict(q_start=4096), dict(q=None), dict(k=4104), dict(v=None),
                                 dict(o=None), dict(lse=None), dict(causal=2), dict(window=1 << 30), dict(seq_k=1 << 30), dict(batch=1 << 23),
                                 dict(q_stride=(2048, 256, 60)), dict(k_stride=(2048, -256, 64)), dict(v_stride=(2048, (1 << 22) + 8, 64)),
                                 dict(k_len=4096, q_start=4096, k_start=4096)])
def test_attention_refuses(bad):
    lib, n = ops._load(), C.c_uint64()
    assert lib.g10_attention_workspace(C.byref(attention_args()), C.byref(n)) == 0
    assert lib.g10_attention_backward_workspace(C.byref(attention_args()), C.byref(n)) == 0 and n.value == 2 * 4 * 8 * 8 + 256
    assert lib.g10_attention(C.byref(attention_args(**bad)), 4096, 1 << 40, None) == binding.EINVAL
    assert lib.g10_attention_backward(C.byref(attention_args(**bad)), 4096, 1 << 40, None) == binding.EINVAL


def test_attention_backward_refuses():
    lib = ops._load()
    for n in ("d_o", "dq", "dk", "dv"):
        assert lib.g10_attention_backward(C.byref(attention_args(**{n: None})), 4096, 1 << 40, None) == binding.EINVAL, n
    assert lib.g10_attention_backward(C.byref(attention_args()), None, 0, None) == binding.EINVAL
    assert lib.g10_attention_backward(C.byref(attention_args()), 4096, 100, None) == binding.EINVAL


def test_adamw_blocks_and_refusals():
    lib, n = ops._load(), C.c_uint64()
    ts = (ops._AdamwTensor * 4)((4096, None, 1), (4096, None, 256), (4096, None, 0), (4096, None, 257))
    assert lib.g10_adamw_blocks(ts, 4, C.byref(n)) == 0 and n.value == 4
    h = C.c_void_p()

    def create(**kw):
        args = dict(tensors=ts, count=4, type=ops.F32, grad_type=ops.F32, copy_type=0, state_type=ops.F32, m=4096, v=4096)
        args.update(kw)
        return lib.g10_adamw_create(C.byref(ops._AdamwDesc(**args)), None, C.byref(h))

    for bad in (dict(type=3), dict(grad_type=9), dict(state_type=ops.BF16), dict(m=None), dict(v=4100), dict(state_type=ops.E4M3),
                dict(tensors=None), dict(count=(1 << 20) + 1)):
        assert create(**bad) == binding.EINVAL, bad
    ts[1].copy = 4096
    assert create() == binding.EINVAL                                  # copies of type float32
    ts[1].copy, ts[0].p = None, 4098
    assert create() == binding.EINVAL
    ts[0].p, ts[0].n = 4096, 1 << 40
    assert create() == binding.EINVAL
    assert not h.value


def test_binding_refuses_what_is_not_on_a_device():
    x = torch.zeros(1, 2, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="GPU memory"):
        ops.g10_attention(x, x, x)
    with pytest.raises(ValueError, match="GPU memory"):
        ops.g10_norm_rope(x, x, torch.zeros(2, 64), torch.zeros(1, 2, dtype=torch.int32))
    with pytest.raises(ValueError, match="GPU memory"):
        ops.AdamW([torch.zeros(3)])
    with pytest.raises(ValueError, match="no parameters"):
        ops.AdamW([])
    with pytest.raises(ValueError, match="even"):
        ops.rope_table(4, 3, device="cpu")


def test_rope_table_far_positions():
    t = ops.rope_table(200001, 64, device="cpu")
    import math
    for pos, i in ((0, 0), (1, 5), (200000, 0), (200000, 1), (131071, 31)):
        a = pos * 10000.0 ** (-2 * i / 64)
        assert abs(float(t[pos, i]) - math.cos(a)) <= 2 ** -24 + 1e-9 and abs(float(t[pos, 32 + i]) - math.sin(a)) <= 2 ** -24 + 1e-9
