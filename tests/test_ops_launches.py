"""What the operators launch, for sizes up to the largest: the library's host code in a process of its own against tests/native/launches.cpp in
place of the HIP runtime (no GPU, kernels do not run).  A launch's work-items are counted in 32 bits."""
import json
import os
import subprocess
import sys

import pytest

from paper_2310_09443_amd import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHILD = r"""
import ctypes as C, json, sys
shim = C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL)                 # before the library: its calls resolve to these
sys.path.insert(0, "tests")
from paper_2310_09443_amd import binding as B, ops
import test_ops_abi as A
lib = C.CDLL(B.LIB_PATH)
shim.test_name.restype = C.c_char_p
shim.test_dim.restype = C.c_uint32
lib.g10_attention.argtypes = lib.g10_attention_backward.argtypes = [C.c_void_p, C.c_void_p, C.c_uint64, C.c_void_p]

def seen(rc):
    # (code, [kernel, workgroups, threads of one])
    out = [[shim.test_name(C.c_long(i)).decode()] + [shim.test_dim(C.c_long(i), b, 0) * shim.test_dim(C.c_long(i), b, 1) * shim.test_dim(C.c_long(i), b, 2) for b in (0, 1)]
           for i in range(shim.test_count())]
    shim.test_clear()
    return [rc, out]

got = []
for kind, kw in json.loads(sys.argv[2]):
    n = C.c_uint64()
    if kind in ("attention", "backward"):
        a = A.attention_args(**kw)
        name = "g10_attention" if kind == "attention" else "g10_attention_backward"
        rc = getattr(lib, name + "_workspace")(C.byref(a), C.byref(n))
        got.append(seen(getattr(lib, name)(C.byref(a), 4096, n.value, None) if rc == 0 else rc) + [n.value])
    elif kind == "rope":
        a = A.rope_args(**kw)
        got.append(seen(lib.g10_norm_rope(C.byref(a), None)) + [0])
    else:
        t = (ops._AdamwTensor * 1)((4096, None, kw["n"]))
        h = C.c_void_p()
        assert lib.g10_adamw_create(C.byref(ops._AdamwDesc(tensors=t, count=1, m=4096, v=4096)), None, C.byref(h)) == 0
        p = ops._AdamwParams(1e-3, 0.9, 0.999, 1e-8, 0.0, 1, None)
        got.append(seen(lib.g10_adamw_step(h, (C.c_void_p * 1)(4096), C.byref(p), None)) + [0])
        lib.g10_adamw_free(h)
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


def fits(launch):
    name, groups, threads = launch
    return 0 < groups and groups * threads < 1 << 32


def packed(batch, rows, heads=32, kv=8, **kw):
    """Sequences of which only the sum of lengths is told."""
    return dict(dict(batch=batch, heads=heads, kv_heads=kv, dim=64, seq_q=rows, seq_k=rows, q_start=4096, k_start=4096, max_q=rows, max_k=rows), **kw)


SIZES = [packed(4096, 4096), packed(65600, 65600), packed(256, 262144, 32, 32), packed(300, 300000, 32, 32), packed(524000, 524000, 32, 1),
         packed(20000, 1 << 29, 32, 32), packed(1, (1 << 30) - 1, 64, 1), packed(2, 1 << 20, max_q=1, max_k=1), packed(1000, 64000, max_q=0, max_k=1 << 29),
         dict(batch=131072, heads=64, kv_heads=64, seq_q=4096, seq_k=4096), dict(batch=70000, heads=32, kv_heads=8, seq_q=1, seq_k=1000),
         dict(batch=8, heads=32, kv_heads=8, seq_q=1, seq_k=32768), dict(batch=3, heads=40, kv_heads=8, seq_q=5, seq_k=(1 << 30) - 1)]


@pytest.mark.parametrize("kind", ["attention", "backward"])
def test_attention_fits_into_its_grid_and_reaches_every_head(launches, kind):
    for kw, (rc, ran, _) in zip(SIZES, launches(*[(kind, kw) for kw in SIZES])):
        assert rc == 0 and ran, kw
        units, heads = kw["batch"] * kw["kv_heads"], kw["batch"] * kw["heads"]
        rest = 64 if "q_start" in kw else 0                            # workgroups that clear rows of no sequence
        for name, groups, threads in ran:
            assert fits((name, groups, threads)), (kw, name, groups)
            round8 = units if units % 8 and units < 64 else (units + 7) // 8 * 8
            if "k_attn_split" in name and groups - rest not in (256, 512):
                assert (groups - rest) % round8 == 0, (kw, name, groups)
            if "k_attn_join" in name:
                assert groups % units == 0, (kw, name, groups)
            if "k_attn_fwd" in name or "k_attn_dq" in name:
                assert (groups - rest) % (round8 * kw["heads"] // kw["kv_heads"]) == 0 and groups - rest >= heads, (kw, name, groups)
            if "k_attn_dkdv" in name and groups - rest not in (256, 512):
                assert (groups - rest) % round8 == 0, (kw, name, groups)


def test_small_grids_are_what_the_work_asks_for(launches):
    (rc, ran, _), = launches(("attention", dict(batch=16, heads=32, kv_heads=32, dim=128, seq_q=2048, seq_k=2048)))
    assert rc == 0 and [x[1:] for x in ran] == [[16 * 32 * 16, 256]]
    (rc, ran, _), = launches(("attention", packed(16, 16 * 2048, 32, 32, max_q=2048, max_k=2048)))
    assert rc == 0 and [x[1:] for x in ran] == [[16 * 32 * 16 + 64, 256]]
    (rc, ran, _), = launches(("attention", packed(8, 8, max_q=1, max_k=1)))
    assert rc == 0 and [x[1:] for x in ran] == [[8 * 8 + 64, 256]]


def test_starts_that_fall_do_not_make_counts_wrap(launches):
    """Work is cut into shares by counts in 32 bits.  Starts such as 0, n, 0, n, ... make every second sequence as long as all rows:
    where their tiles together could pass 2^31, nothing is cut, and the few-query kernel has nothing to count."""
    calls = [packed(256, 1024, 8, 1, seq_k=1 << 22), packed(200, 1600, 8, 2, seq_k=1 << 24), packed(100, 100, 32, 8, seq_k=10_000_000), packed(8, 8, 32, 8, seq_k=8 * 32768)]
    for kw, cut, (rc, ran, n) in zip(calls, (False, False, True, True), launches(*[("attention", kw) for kw in calls])):
        tiles = (kw["batch"] + 1) // 2 * -(-kw["seq_q"] * kw["heads"] // kw["kv_heads"] // 32) * kw["kv_heads"] * (kw["seq_k"] // 32)
        assert rc == 0 and (tiles < 1 << 31) == cut and any("k_attn_join" in x[0] for x in ran) == cut == (n > 0), (kw, ran)


def test_more_heads_than_a_grid_has_workgroups_are_refused(launches):
    for kw in (dict(batch=1 << 22, heads=4), dict(batch=1 << 18, heads=64, kv_heads=64), dict(batch=1 << 24, heads=2, kv_heads=1)):
        for rc, ran, _ in launches(("attention", kw), ("backward", kw)):
            assert rc == -1 and not ran, kw


def test_norm_and_rotation_of_many_rows(launches):
    calls = [("rope", dict(batch=1 << 20, seq=64, dim=100, rot=100)), ("rope", dict(batch=1 << 15, seq=1 << 20, dim=8, rot=0)), ("rope", dict(batch=3, seq=5))]
    for call, (rc, ran, _) in zip(calls, launches(*calls)):
        assert rc == 0 and len(ran) == 1 and fits(ran[0]), (call, ran)


def test_weights_of_many_chunks(launches):
    chunks = (1 << 24) + 5
    (rc, ran, _), (rc1, one, _) = launches(("adamw", dict(n=chunks * 2048)), ("adamw", dict(n=5000)))
    assert rc == 0 and all(fits(x) for x in ran) and sum(x[1] for x in ran) == chunks
    assert rc1 == 0 and [x[1] for x in one] == [3]
