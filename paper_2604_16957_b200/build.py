"""Build libtq.so (the C-ABI CUDA library) in-tree with nvcc for sm_100a, then the serving operators' Python binding.

    python -m paper_2604_16957_b200.build [--force] [--verbose]
    python -m paper_2604_16957_b200.build --probe copies|math    # timing-probe builds of the decode kernel

The probe libraries (libtq_probe_copies.so, libtq_probe_math.so) are the same sources compiled with
-DTQ_PROBE_COPIES_ONLY / -DTQ_PROBE_MATH_ONLY: the fused decode kernel with its arithmetic, or its copies,
taken out.  They produce meaningless results and exist only to time (`bench.py --lib <path>`).
"""
import glob
import os
import re
import subprocess
import sys
import sysconfig
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")
LIB = os.path.join(HERE, "libtq.so")

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    # bit-exact quantiser: IEEE division / sqrt, no flush-to-zero, no fast-math; FMA contraction
    # is harmless because every quantiser operation is an explicit _rn intrinsic
    "-prec-div=true", "-prec-sqrt=true", "-ftz=false",
    "-Xcompiler", "-fPIC", "-shared", "-cudart", "static",
]


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def _stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = sources() + glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(os.path.join(INCLUDE, "*.h"))
    return any(os.path.getmtime(p) > t for p in deps)


def binding_path() -> str:
    """Native binding of the serving operators: a CPython extension of this torch, its C++ ABI and this Python, all of which
    its name tells, so that one made for others is neither loaded nor taken for up to date."""
    import torch
    made_for = re.sub(r"[^0-9A-Za-z.]", "_", f"torch{torch.__version__}_abi{int(torch._C._GLIBCXX_USE_CXX11_ABI)}")
    return os.path.join(HERE, f"_tq_bind.{made_for}{sysconfig.get_config_var('EXT_SUFFIX')}")


def build_binding(force: bool = False) -> str:
    """The extension that hands torch tensors to libtq; needs g++ and torch's headers, no CUDA compiler."""
    src, out = os.path.join(CSRC, "binding", "tq_bind.cpp"), binding_path()
    if not force and os.path.exists(out) and all(os.path.getmtime(p) <= os.path.getmtime(out)
                                                 for p in [src] + glob.glob(os.path.join(INCLUDE, "*.h"))):
        return out
    import torch
    from torch.utils import cpp_extension
    cuda = os.path.dirname(os.path.dirname(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")))
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}"]
    for path in cpp_extension.include_paths() + [os.path.join(cuda, "include"), sysconfig.get_paths()["include"]]:
        cmd += ["-isystem", path]
    lib = os.path.join(os.path.dirname(torch.__file__), "lib")
    made = f"{out}.{os.getpid()}.tmp"  # a process that has the old one loaded keeps it
    cmd += ["-I", INCLUDE, src, "-o", made, "-L", lib, "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda"]
    try:
        subprocess.run(cmd, check=True)
        os.replace(made, out)
    finally:
        if os.path.exists(made):
            os.remove(made)
    return out


def build(force: bool = False, verbose: bool = False) -> str:
    if force or _stale():
        build_library(verbose)
    build_binding(force)
    return LIB


def build_library(verbose: bool = False) -> str:
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    extra = ["-Xptxas", "-v"] if verbose else []
    with tempfile.TemporaryDirectory() as tmp:  # one nvcc per source file, side by side
        def compile_one(src):
            obj = os.path.join(tmp, os.path.basename(src) + ".o")
            subprocess.run([nvcc] + NVCC_FLAGS[:-3] + extra + ["-I", INCLUDE, "-I", CSRC, "-c", src, "-o", obj], check=True)
            return obj

        with ThreadPoolExecutor(max(1, min(8, os.cpu_count() or 1))) as pool:
            objects = list(pool.map(compile_one, sources()))
        subprocess.run([nvcc] + NVCC_FLAGS + ["-o", LIB] + objects, check=True)
    return LIB


def build_probe(which: str) -> str:
    """Timing-probe build of the library: which = "copies" or "math"."""
    macro = {"copies": "TQ_PROBE_COPIES_ONLY", "math": "TQ_PROBE_MATH_ONLY"}[which]
    out = os.path.join(HERE, f"libtq_probe_{which}.so")
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    subprocess.run([nvcc] + NVCC_FLAGS + ["-D" + macro, "-I", INCLUDE, "-I", CSRC, "-o", out] + sources(), check=True)
    return out


if __name__ == "__main__":
    if "--probe" in sys.argv:
        print(build_probe(sys.argv[sys.argv.index("--probe") + 1]))
    else:
        print(build(force="--force" in sys.argv, verbose="--verbose" in sys.argv))
