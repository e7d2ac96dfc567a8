"""Entry points of the operators around attention: structs as the header has them, what is refused before anything reaches a device, and what is
launched for sizes up to the largest (without a GPU: tests/native/launches.cpp in place of the HIP runtime)."""
import ctypes as C
import json
import os
import subprocess
import sys

import pytest
import torch

from paper_2310_09443_amd import binding, build, ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STRUCTS = {"g10_embed_args": "_Embed", "g10_norm_args": "_Norm", "g10_log_probs_args": "_LogProbs", "g10_gated_args": "_Gated"}


def test_struct_layouts_match_the_header(tmp_path):
    lines = []
    for c, py in STRUCTS.items():
        lines.append(f'printf("{c} %zu", sizeof({c}));')
        for f, _ in getattr(ops, py)._fields_:
            lines.append(f'printf(" %zu", offsetof({c}, {f}));')
        lines.append('puts("");')
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "g10_ops.h"\nint main(void) {\n' + "\n".join(lines) + "\nreturn 0;\n}\n")
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    for line in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.splitlines():
        name, *n = line.split()
        t = getattr(ops, STRUCTS[name])
        assert [int(x) for x in n] == [C.sizeof(t)] + [getattr(t, f).offset for f, _ in t._fields_], name


def fill(t, **kw):
    a = t()
    for n, x in kw.items():
        setattr(a, n, x)
    return a


def embed_args(**kw):
    return fill(ops._Embed, **dict(dict(ids=4096, table=4096, out=4096, dout=4096, dtable=4096, table_stride=64, out_stride=64, dout_stride=64, dtable_stride=64,
                                        tokens=10, vocab=100, dim=64, scale=1.0, type=ops.BF16), **kw))


def norm_args(**kw):
    return fill(ops._Norm, **dict(dict(x=4096, dy=4096, weight=4096, bias=4096, out=4096, dweight=4096, dbias=4096, x_stride=64, dy_stride=64, out_stride=64, rows=10,
                                       dim=64, eps=1e-6, center=1, type=ops.BF16, weight_type=ops.BF16), **kw))


def log_probs_args(**kw):
    return fill(ops._LogProbs, **dict(dict(logits=4096, tokens=4096, logp=4096, lse=4096, entropy=4096, top_logp=4096, top_ids=4096, dlogp=4096, dentropy=4096,
                                           dlogits=4096, logits_stride=100, dlogits_stride=100, rows=10, vocab=100, top=5, scale=1.0, ignore=-100, type=ops.BF16), **kw))


def gated_args(**kw):
    return fill(ops._Gated, **dict(dict(x=4096, gate=4096, up=4096, h=4096, dh=4096, dx=4096, dgate=4096, dup=4096, x_stride=64, gate_stride=128, up_stride=128, h_stride=128, dh_stride=128,
                                        dx_stride=64, dw_stride=128, tokens=10, dim=64, inner=128, act=ops.SILU, type=ops.BF16), **kw))


MAKE = {"g10_embed": embed_args, "g10_embed_backward": embed_args, "g10_norm": norm_args, "g10_norm_backward": norm_args, "g10_log_probs": log_probs_args,
        "g10_log_probs_backward": log_probs_args, "g10_gated": gated_args, "g10_gated_backward": gated_args}


def call(lib, name, a, room=1 << 60):
    f = getattr(lib, name)
    return f(a, 4096, room, None) if len(f.argtypes) == 4 else f(a, None)


def test_null_arguments_are_refused():
    lib = ops._load()
    for name, make in MAKE.items():
        assert call(lib, name, None) == binding.EINVAL
        if hasattr(lib, name + "_workspace") and len(getattr(lib, name).argtypes) == 4:
            f, n = getattr(lib, name + "_workspace"), C.c_uint64()
            assert f(None, C.byref(n)) == binding.EINVAL and f(C.byref(make()), None) == binding.EINVAL and f(C.byref(make()), C.byref(n)) == 0


BOTH = [("embed", dict(type=3)), ("embed", dict(dim=0)), ("embed", dict(dim=65537)), ("embed", dict(vocab=0)), ("embed", dict(vocab=1 << 31)), ("embed", dict(tokens=1 << 31)),
        ("embed", dict(scale=float("nan"))), ("embed", dict(scale=float("inf"))), ("embed", dict(ids=None)), ("embed", dict(ids=4098)), ("embed", dict(ids_64=2)),
        ("embed", dict(ids_64=1, ids=4100)),
        ("norm", dict(type=3)), ("norm", dict(weight_type=ops.F16)), ("norm", dict(dim=0)), ("norm", dict(dim=65537)), ("norm", dict(rows=1 << 31)), ("norm", dict(eps=-1.0)),
        ("norm", dict(eps=float("nan"))), ("norm", dict(eps=float("inf"))), ("norm", dict(center=2)), ("norm", dict(x=None)), ("norm", dict(out=None)), ("norm", dict(x=4097)),
        ("norm", dict(weight=4097)), ("norm", dict(weight_type=ops.F32, bias=4098)),
        ("log_probs", dict(type=3)), ("log_probs", dict(scale=0.0)), ("log_probs", dict(scale=float("nan"))), ("log_probs", dict(scale=float("inf"))),
        ("log_probs", dict(vocab=0)), ("log_probs", dict(vocab=1 << 31)), ("log_probs", dict(rows=1 << 31)), ("log_probs", dict(logits=None)), ("log_probs", dict(lse=None)),
        ("log_probs", dict(logits=4097)), ("log_probs", dict(tokens=4100)),
        ("gated", dict(type=ops.F32)), ("gated", dict(act=2)), ("gated", dict(out_in=2)), ("gated", dict(dim=0)), ("gated", dict(dim=(1 << 20) + 8)), ("gated", dict(tokens=1 << 31)), ("gated", dict(x=None)), ("gated", dict(gate=4097)), ("gated", dict(up=None)),
        ("gated", dict(x_stride=56)), ("gated", dict(up_stride=127)), ("gated", dict(gate_stride=-128)), ("gated", dict(out_in=1, gate_stride=56))]


@pytest.mark.parametrize("op, bad", BOTH)
def test_both_passes_refuse(op, bad):
    lib = ops._load()
    for name in ("g10_" + op, f"g10_{op}_backward"):
        assert call(lib, name, C.byref(MAKE[name](**bad))) == binding.EINVAL


@pytest.mark.parametrize("name, bad", [("embed", dict(table=None)), ("embed", dict(out=None)), ("embed", dict(out=4097)), ("embed_backward", dict(dout=None)),
                                       ("embed_backward", dict(dtable=None)), ("embed_backward", dict(dtable=None, tokens=0)), ("embed_backward", dict(dout=4097)),
                                       ("norm_backward", dict(dy=None)), ("norm_backward", dict(dy=4097)), ("norm_backward", dict(weight=None)),
                                       ("norm_backward", dict(dweight=4097)), ("log_probs", dict(top=65)), ("log_probs", dict(top=5, vocab=4)),
                                       ("log_probs", dict(logp=None)), ("log_probs", dict(top_ids=None)), ("log_probs", dict(top_logp=None)),
                                       ("log_probs_backward", dict(dlogits=None)), ("log_probs_backward", dict(tokens=None)), ("log_probs_backward", dict(entropy=None)),
                                       ("log_probs_backward", dict(dlogits=4097)), ("gated", dict(h=None)), ("gated", dict(h_stride=120)), ("gated_backward", dict(dh=4097)),
                                       ("gated_backward", dict(dx=None)), ("gated_backward", dict(dgate=None)), ("gated_backward", dict(dup=4101)),
                                       ("gated_backward", dict(dw_stride=120)), ("gated_backward", dict(dx_stride=60))])
def test_one_pass_refuses(name, bad):
    assert call(ops._load(), "g10_" + name, C.byref(MAKE["g10_" + name](**bad))) == binding.EINVAL


def test_workspaces_are_needed():
    lib, n = ops._load(), C.c_uint64()
    for name in ("g10_embed_backward", "g10_norm_backward", "g10_gated_backward"):
        a = MAKE[name]()
        assert getattr(lib, name + "_workspace")(C.byref(a), C.byref(n)) == 0 and n.value > 0
        assert getattr(lib, name)(C.byref(a), None, n.value, None) == binding.EINVAL
        assert getattr(lib, name)(C.byref(a), 4096, n.value - 1, None) == binding.EINVAL
        assert getattr(lib, name)(C.byref(a), 4097, n.value, None) == binding.EINVAL


def test_calls_on_host_tensors_are_refused():
    x, w, ids = torch.zeros(4, 16, dtype=torch.bfloat16), torch.zeros(16, 32, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int64)
    for bad in (lambda: ops.embed(ids, x), lambda: ops.norm(x), lambda: ops.gated(x, w, w), lambda: ops.log_probs(x, ids), lambda: ops.g10_embed_backward(x, ids, 5),
                lambda: ops.g10_norm_backward(x, x), lambda: ops.g10_gated_backward(x, x, w, w), lambda: ops.g10_log_probs_backward(ids, x, ids, ids)):
        with pytest.raises(ValueError, match="GPU memory"):
            bad()


CHILD = r"""
import ctypes as C, json, sys
shim = C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL)                 # before the library: its calls resolve to these
sys.path.insert(0, "tests")
from paper_2310_09443_amd import binding as B, ops
import test_layer_abi as A
lib = C.CDLL(B.LIB_PATH)
shim.test_name.restype = C.c_char_p
shim.test_dim.restype = C.c_uint32
got = []
for name, kw in json.loads(sys.argv[2]):
    a, n = A.MAKE[name](**kw), C.c_uint64()
    room = name not in ("g10_embed", "g10_norm", "g10_log_probs_backward")
    rc = getattr(lib, name + "_workspace")(C.byref(a), C.byref(n)) if room else 0
    if rc == 0:
        rc = getattr(lib, name)(C.byref(a), C.c_void_p(4096), n, None) if room else getattr(lib, name)(C.byref(a), None)
    got.append([rc, [[shim.test_name(C.c_long(i)).decode()] + [shim.test_dim(C.c_long(i), b, 0) * shim.test_dim(C.c_long(i), b, 1) * shim.test_dim(C.c_long(i), b, 2)
                     for b in (0, 1)] for i in range(shim.test_count())], n.value])
    shim.test_clear()
print(json.dumps(got))
"""


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    if not os.path.exists(build.LIB):
        build.build()
    shim = str(tmp_path_factory.mktemp("shim") / "launches.so")
    subprocess.run(["g++", "-O1", "-std=c++17", "-fPIC", "-shared", os.path.join(ROOT, "tests", "native", "launches.cpp"), "-o", shim], check=True)

    def run(*calls):
        r = subprocess.run([sys.executable, "-c", CHILD, shim, json.dumps(calls)], cwd=ROOT, capture_output=True, text=True, timeout=300)
        assert r.returncode == 0, r.stderr[-2000:]
        return json.loads(r.stdout.strip().splitlines()[-1])
    return run


BIG = (1 << 31) - 1


def test_largest_sizes_fit_into_their_grids(launches):
    calls = [("g10_embed", dict(tokens=BIG, dim=8)), ("g10_embed", dict(tokens=BIG, dim=65535)), ("g10_embed_backward", dict(tokens=BIG, vocab=BIG, dim=8)),
             ("g10_embed_backward", dict(tokens=0, vocab=BIG)), ("g10_norm", dict(rows=BIG, dim=8)), ("g10_norm_backward", dict(rows=BIG, dim=65536)),
             ("g10_log_probs", dict(rows=BIG, vocab=100)), ("g10_log_probs", dict(rows=3, vocab=BIG)), ("g10_log_probs_backward", dict(rows=BIG)),
             ("g10_gated", dict(tokens=1 << 24, inner=1 << 10, gate_stride=1 << 10, up_stride=1 << 10, h_stride=1 << 10)),
             ("g10_gated_backward", dict(tokens=1 << 22, inner=1 << 10, gate_stride=1 << 10, up_stride=1 << 10, dh_stride=1 << 10, dw_stride=1 << 10))]
    for c, (rc, ran, n) in zip(calls, launches(*calls)):
        assert rc == 0 and ran, c
        for name, groups, threads in ran:
            assert 0 < groups and groups * threads < 1 << 32, (c, name, groups)


def test_more_tiles_than_a_grid_holds_are_refused(launches):
    kw = dict(dim=8, inner=1 << 20, gate_stride=1 << 20, up_stride=1 << 20, h_stride=1 << 20, x_stride=8)
    (rc, ran, _), (rc1, ran1, _) = launches(("g10_gated", dict(tokens=BIG, **kw)), ("g10_gated", dict(tokens=4096, **kw)))
    assert rc == binding.EINVAL and not ran and rc1 == 0 and len(ran1) == 1


def test_no_rows_launch_nothing_but_what_clears_gradients(launches):
    calls = [("g10_embed", dict(tokens=0)), ("g10_norm", dict(rows=0)), ("g10_log_probs", dict(rows=0)), ("g10_log_probs_backward", dict(rows=0)), ("g10_gated", dict(tokens=0)),
             ("g10_embed_backward", dict(tokens=0)), ("g10_norm_backward", dict(rows=0)), ("g10_gated_backward", dict(tokens=0))]
    got = launches(*calls)
    assert all(rc == 0 for rc, _, _ in got) and [len(ran) for _, ran, _ in got] == [0] * 5 + [1] * 3, got


def test_every_tile_has_a_workgroup(launches):
    """Of a product's tiles, their rows by their columns by the shares of the sum (or the products side by side)."""
    sizes = [(1, 64, 128), (32, 4096, 16384), (33, 4096, 16384), (5001, 1000, 2744), (8192, 4096, 16384), (100, 8, 8), (300, 12000, 64)]
    for out_in in (0, 1):
        calls = [("g10_gated", dict(tokens=m, dim=k, inner=n, out_in=out_in, x_stride=k, gate_stride=k if out_in else n, up_stride=k if out_in else n, h_stride=n)) for m, k, n in sizes]
        for (m, k, n), (rc, ran, room) in zip(sizes, launches(*calls)):
            assert rc == 0 and "k_gated" in ran[0][0], (m, k, n)
            shares = room // (m * 2 * n * 4) or 1
            assert len(ran) == (2 if shares > 1 else 1) and room == (shares * m * 2 * n * 4 if shares > 1 else 0)
            tiles = [-(-m // rows) * -(-n // wide) * shares for rows, wide in ((256, 128), (128, 128), (64, 128), (64, 64))]
            assert any(t <= ran[0][1] < t + 8 for t in tiles), (m, k, n, ran)


def test_every_cut_of_tiles_is_reached(launches):
    """Large products, middling ones, few tokens on large weights and on small ones; sums in shares and whole."""
    sizes = [(8192, 4096, 16384), (16384, 768, 2048), (2048, 1024, 2816), (300, 512, 2048), (64, 4096, 16384), (8, 4096, 16384), (16, 512, 2048), (100, 4096, 4096)]
    seen = set()
    for out_in in (0, 1):
        for name, more in (("g10_gated", {}), ("g10_gated_backward", {})):
            calls = [(name, dict(tokens=m, dim=k, inner=n, out_in=out_in, x_stride=k, dx_stride=k, gate_stride=k if out_in else n, up_stride=k if out_in else n, dw_stride=k if out_in else n, h_stride=n, dh_stride=n))
                     for m, k, n in sizes]
            for rc, ran, _ in launches(*calls):
                assert rc == 0
                seen |= {x[0] for x in ran}
    cuts = {tuple(part for part in ("Li2ELi4ELi4ELi64ELi2", "Li1ELi4ELi4ELi32ELi3", "Li1ELi4ELi2ELi64ELi2", "Li2ELi2ELi1ELi64ELi6") if part in x) for x in seen if "join" not in x}
    assert cuts == {("Li2ELi4ELi4ELi64ELi2",), ("Li1ELi4ELi4ELi32ELi3",), ("Li1ELi4ELi2ELi64ELi2",), ("Li2ELi2ELi1ELi64ELi6",)} and any("join" in x for x in seen), seen
