"""Builds the HIP libraries in-tree for gfx950 with hipcc (cross-compiles without a GPU)."""
from __future__ import annotations

import os
import re
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
HIP_FLAGS = ["-O3", "--offload-arch=gfx950", "-std=c++17", "-shared", "-fPIC",
             "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-Wno-unused-command-line-argument",
             "-Werror=align-mismatch"]

LIBCADA = os.path.join(HERE, "libcada.so")
LIBCADA_SRC = [os.path.join(HERE, "csrc", f) for f in
               ("cada_api.hip", "cada_logreg.hip", "cada_logreg_fused.hip", "cada_logreg_small.hip", "cada_logreg_steps.hip", "cada_logreg_rows.hip", "cada_server.hip",
                "cada_mlp.hip", "cada_mlp_eval.hip", "cada_linear.hip", "cada_linear_xent.hip", "cada_norm.hip", "cada_embedding.hip", "cada_xent.hip", "cada_adamw.hip")]


def _run(cmd):
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    out = "\n".join(l for l in r.stdout.splitlines() if "packed-fp32-ops" not in l and not re.fullmatch(r"\d+ warnings? generated.*", l))
    if r.returncode != 0:
        raise RuntimeError("build failed: %s\n%s" % (" ".join(cmd), out))
    if out:
        print(out, file=sys.stderr, flush=True)      # warnings
    return out


def build_libcada() -> str:
    """Compiles the translation units side by side (objects in a temporary folder), then links."""
    import tempfile
    from concurrent.futures import ThreadPoolExecutor
    compile_flags = [f for f in HIP_FLAGS if f != "-shared"] + ["-c", "-I", os.path.join(ROOT, "include")]
    with tempfile.TemporaryDirectory(prefix="libcada_build_") as tmp:
        objs = [os.path.join(tmp, os.path.basename(src) + ".o") for src in LIBCADA_SRC]
        with ThreadPoolExecutor(max_workers=min(len(objs), os.cpu_count() or 1)) as pool:
            list(pool.map(lambda so: _run([HIPCC, *compile_flags, "-o", so[1], so[0]]), zip(LIBCADA_SRC, objs)))
        _run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIBCADA, *objs])
    return LIBCADA


OPS_BINDING = os.path.join(HERE, "_ops.so")


def build_ops_binding() -> str:
    """The Python module of the operators (host code on torch's C++ tensors), next to libcada.so, which it links to."""
    import sysconfig
    import torch
    from torch.utils.cpp_extension import include_paths, library_paths
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch._C._GLIBCXX_USE_CXX11_ABI,
           "-I", os.path.join(ROOT, "include"), "-isystem", sysconfig.get_paths()["include"]]
    for p in include_paths():
        cmd += ["-isystem", p]
    cmd += ["-o", OPS_BINDING, os.path.join(HERE, "csrc", "ops_binding.cpp"), "-L", HERE, "-l:libcada.so", "-Wl,-rpath,$ORIGIN"]
    for p in library_paths():
        cmd += ["-L", p]
    _run(cmd + ["-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10"])
    return OPS_BINDING


def ops_binding_lacks() -> str:
    """What the operators' Python module needs and is not here (torch with its C++ headers, Python's headers, a host compiler), or an empty text."""
    import shutil
    import sysconfig
    try:
        from torch.utils.cpp_extension import include_paths
    except ImportError:
        return "torch"
    if not any(os.path.exists(os.path.join(p, "ATen", "ATen.h")) for p in include_paths()):
        return "torch's C++ headers"
    if not os.path.exists(os.path.join(sysconfig.get_paths()["include"], "Python.h")):
        return "Python's headers"
    cxx = os.environ.get("CXX", "g++")
    return "" if shutil.which(cxx.split()[0]) else "a host compiler (%s)" % cxx


def build_all() -> None:
    build_libcada()
    build_ops_binding()


def main() -> int:
    """libcada.so, which the C ABI is all of, and the operators' Python module where what that needs is here."""
    build_libcada()
    print("built", LIBCADA)
    lacks = ops_binding_lacks()
    if lacks:
        print("not built: %s, which needs %s (the C ABI does not need it)" % (OPS_BINDING, lacks), file=sys.stderr)
    else:
        build_ops_binding()
        print("built", OPS_BINDING)
    return 0


if __name__ == "__main__":
    sys.exit(main())
