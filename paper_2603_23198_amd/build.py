"""Build libsfl.so (HIP kernels for gfx950 + the C ABI) in-tree with hipcc, and the
binding's `_marshal.so` (tensors to checked pointers) with the host compiler.

Every source under csrc/ is compiled to an object file in parallel, then linked
into `libsfl.so` next to this file. The build always recompiles (it is the
"does it build" check); `python -m paper_2603_23198_amd.build` runs it.
"""
from __future__ import annotations

import concurrent.futures as cf
import contextlib
import glob
import os
import shutil
import subprocess
import sys
import sysconfig
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libsfl.so")
MARSHAL = os.path.join(HERE, "_marshal.so")
ARCH = "gfx950"  # the kernels use CDNA4 instructions (MFMA 16x16x32 bf16, ds_read_b64_tr_b16)

FLAGS = [
    "-O3", "-std=c++17", "-fPIC", f"--offload-arch={ARCH}",
    # keep the compiler from emitting packed fp32 arithmetic (v_pk_* f32)
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-munsafe-fp-atomics",
    # the GEMM epilogues index their accumulator arrays from fully unrolled loops; let the
    # unroller expand them however large, so the arrays stay in registers
    "-mllvm", "-pragma-unroll-threshold=1000000",
    "-Wno-unused-result",
]


def hipcc():
    for c in (os.environ.get("HIPCC"), shutil.which("hipcc"), "/opt/rocm/bin/hipcc"):
        if c and os.path.exists(c):
            return c
    raise RuntimeError("hipcc not found")


def _compile(src, obj, extra=()):
    cmd = [hipcc(), *FLAGS, *extra, "-x", "hip", "-c", src, "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    errs = "\n".join(l for l in (r.stderr or "").splitlines() if "packed-fp32-ops" not in l)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed for {os.path.basename(src)}:\n{errs}")
    return errs


@contextlib.contextmanager
def _beside(path):
    """A temporary name beside `path`, to be moved there when it is complete."""
    tmp = path + ".tmp"
    try:
        yield tmp
    finally:
        if os.path.exists(tmp):
            os.remove(tmp)


def _compile_marshal(out):
    import torch
    at = os.path.dirname(torch.__file__)
    cxx = shutil.which("g++") or shutil.which("c++") or hipcc()
    cmd = [cxx, "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}",
           "-I", sysconfig.get_paths()["include"], "-isystem", os.path.join(at, "include"),
           "-isystem", os.path.join(at, "include", "torch", "csrc", "api", "include"),
           os.path.join(CSRC, "python", "marshal.cpp"), "-L", os.path.join(at, "lib"), "-ltorch_python", "-ltorch_cpu",
           "-lc10", "-Wl,-rpath," + os.path.join(at, "lib"), "-o", out]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"compiling marshal.cpp failed:\n{r.stderr}")


def build_marshal() -> str:
    """Compile the binding's extension module against the installed torch (host code only)."""
    with _beside(MARSHAL) as tmp:
        _compile_marshal(tmp)
        os.replace(tmp, MARSHAL)
    return MARSHAL


def build(verbose=False, jobs=None, extra_flags=(), out=None, csrc=None) -> str:
    """Compile and link; `extra_flags` go to every hipcc line, `out` overrides the library
    path and `csrc` the source directory. Nothing is replaced unless everything was built."""
    lib = out or LIB
    src_dir = csrc or CSRC
    srcs = sorted(glob.glob(os.path.join(src_dir, "*.hip")) + glob.glob(os.path.join(src_dir, "*.cpp")))
    jobs = jobs or min(len(srcs), max(1, (os.cpu_count() or 4)), 16)
    with tempfile.TemporaryDirectory(prefix="sfl_build_") as tmp, _beside(lib) as tmp_lib, \
            _beside(MARSHAL) as tmp_marshal, cf.ThreadPoolExecutor(1) as side:
        marshal = side.submit(_compile_marshal, tmp_marshal) if out is None else None
        objs = [os.path.join(tmp, os.path.basename(s) + ".o") for s in srcs]
        with cf.ThreadPoolExecutor(jobs) as ex:
            for src, msg in zip(srcs, ex.map(lambda a, o: _compile(a, o, extra_flags), srcs, objs)):
                if verbose and msg.strip():
                    print(f"[{os.path.basename(src)}]\n{msg}", file=sys.stderr)
        cmd = [hipcc(), f"--offload-arch={ARCH}", "-shared", "-fPIC", *objs, "-o", tmp_lib]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"link failed:\n{r.stderr}")
        if marshal:
            marshal.result()
            os.replace(tmp_marshal, MARSHAL)
        os.replace(tmp_lib, lib)
    return lib


if __name__ == "__main__":
    print(build(verbose=True))
