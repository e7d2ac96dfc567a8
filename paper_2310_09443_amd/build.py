"""Builds the HIP library for gfx950 into paper_2310_09443_amd/libg10.so, and the marshalling of torch tensors beside it."""
import os
import subprocess
import sysconfig
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
SRC = [os.path.join(HERE, "csrc", f) for f in ("g10_api.hip", "g10_mem.hip", "g10_vitality.hip", "g10_plan.hip", "g10_loop.hip", "g10_prefetch.hip", "g10_replay.hip",
                                               "g10_rope.hip", "g10_attn.hip", "g10_attn_split.hip", "g10_attn_back.hip", "g10_adamw.hip")]
DEPS = SRC + [os.path.join(HERE, "csrc", "g10_internal.h"), os.path.join(HERE, "csrc", "g10_plan_defs.h"), os.path.join(HERE, "csrc", "g10_attn.h"),
              os.path.join(ROOT, "include", "g10.h"), os.path.join(ROOT, "include", "g10_ops.h")]
LIB = os.path.join(HERE, "libg10.so")
TORCH_SRC, TORCH_LIB = os.path.join(HERE, "csrc", "g10_torch.cpp"), os.path.join(HERE, "_g10_torch.so")     # marshalling of torch tensors, host code


def up_to_date() -> bool:
    both = os.path.exists(LIB) and os.path.exists(TORCH_LIB)
    return both and all(os.path.getmtime(LIB) >= os.path.getmtime(d) for d in DEPS) and \
        all(os.path.getmtime(TORCH_LIB) >= os.path.getmtime(d) for d in (TORCH_SRC, os.path.join(ROOT, "include", "g10_ops.h")))


def build_torch() -> str:
    import torch
    from torch.utils.cpp_extension import include_paths
    lib = os.path.join(os.path.dirname(torch.__file__), "lib")
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", "-D__HIP_PLATFORM_AMD__", "-DTORCH_EXTENSION_NAME=_g10_torch",
           "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch._C._GLIBCXX_USE_CXX11_ABI, "-I", os.path.join(ROOT, "include")]
    for p in include_paths() + ["/opt/rocm/include", sysconfig.get_paths()["include"]]:
        cmd += ["-isystem", p]
    subprocess.run(cmd + [TORCH_SRC, "-o", TORCH_LIB, "-L" + lib, "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10", "-lc10_hip"], check=True)
    return TORCH_LIB


def build(force: bool = True) -> str:
    if not force and up_to_date():
        return LIB
    flags = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
             "-I", os.path.join(ROOT, "include"), "-I", os.path.join(HERE, "csrc"), "-Wall", "-Wno-unused-function"]
    with tempfile.TemporaryDirectory() as tmp:                       # one compiler a source, side by side
        objs = [os.path.join(tmp, os.path.basename(f) + ".o") for f in SRC]
        with ThreadPoolExecutor(max_workers=4) as ex:
            host = ex.submit(build_torch)
            list(ex.map(lambda so: subprocess.run(["hipcc"] + flags + ["-c", so[0], "-o", so[1]], check=True), zip(SRC, objs)))
            host.result()
        subprocess.run(["hipcc", "--offload-arch=gfx950", "-fPIC", "-shared"] + objs + ["-o", LIB], check=True)
    return LIB


if __name__ == "__main__":
    print(build(force=True))
