"""Builds libsparsecomm.so (the C-ABI library of sm_100a kernels) in-tree with nvcc."""
from __future__ import annotations

import importlib.util
import os
import shutil
import subprocess
import sys
import sysconfig
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libsparsecomm.so")
SOURCES = ["sc_api.cu", "sc_layer.cu", "sc_norm.cu", "sc_quantized.cu"]
# the layer operators' calls without ctypes; the binding does without where Python's headers are not installed, and without the calls that
# take tensors where torch's are not, or do not compile
CALLS_SOURCE = os.path.join(CSRC, "sc_calls.cpp")
CALLS = os.path.join(HERE, "_sc_calls" + (sysconfig.get_config_var("EXT_SUFFIX") or ".so"))


def _dependencies():
    """Every file under csrc/ plus the public header."""
    deps = [os.path.join(CSRC, f) for f in sorted(os.listdir(CSRC)) if f.endswith((".cu", ".cuh", ".h", ".cpp"))]
    deps.append(os.path.join(HERE, "..", "include", "sparsecomm.h"))
    deps.append(os.path.abspath(__file__))
    return deps


NVCC_FLAGS = [
    "-O3", "-std=c++17", "-lineinfo",
    "-gencode", "arch=compute_100a,code=sm_100a",
    "-Xcompiler", "-fPIC",
    # bit-exact fp32: no fast-math, denormals kept, IEEE division and square root
    "-ftz=false", "-prec-div=true", "-prec-sqrt=true",
]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found: the CUDA library cannot be built")


def _python_headers() -> str:
    return sysconfig.get_paths()["include"]


def _torch_home() -> str:
    spec = importlib.util.find_spec("torch")
    return os.path.dirname(spec.origin) if spec and spec.origin else ""


def _cxx():
    return shutil.which("g++") or shutil.which("c++")


def _calls_wanted() -> bool:
    return os.path.exists(os.path.join(_python_headers(), "Python.h")) and _cxx() is not None


def _calls_commands() -> list:
    """Commands that make the compiled caller, the preferred one first."""
    plain = [_cxx(), "-O2", "-std=c++17", "-shared", "-fPIC", "-I", _python_headers(), "-o", CALLS, CALLS_SOURCE]
    home = _torch_home()
    include, lib = os.path.join(home, "include"), os.path.join(home, "lib")
    if not os.path.exists(os.path.join(include, "torch", "csrc", "autograd", "python_variable.h")):
        return [plain]
    return [plain + ["-DSC_TENSORS", "-I", include, "-I", os.path.join(include, "torch", "csrc", "api", "include"), "-L", lib, "-lc10", "-ltorch_cpu", "-ltorch_python"],
            plain]


def _caller_is_current() -> bool:
    """The compiled caller is not older than its sources; it may be missing where it cannot be built."""
    if not os.path.exists(CALLS):
        return not _calls_wanted()
    sources = (CALLS_SOURCE, os.path.join(HERE, "..", "include", "sparsecomm.h"))
    return all(os.path.getmtime(CALLS) >= os.path.getmtime(d) for d in sources)


def needs_build() -> bool:
    if not os.path.exists(LIB) or not _caller_is_current():
        return True
    t = os.path.getmtime(LIB)
    return any(os.path.getmtime(d) > t for d in _dependencies())


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not needs_build():
        return LIB
    # a caller built from other declarations must not outlive a build that ends without one
    if os.path.exists(CALLS):
        os.remove(CALLS)
    said, failed = [], ""
    # one nvcc per translation unit, side by side, then the link
    with tempfile.TemporaryDirectory(prefix="sparsecomm_build_") as tmp:
        objects = [os.path.join(tmp, os.path.splitext(src)[0] + ".o") for src in SOURCES]
        flags = [_nvcc()] + NVCC_FLAGS
        jobs = [subprocess.Popen(flags + (["-Xptxas", "-v"] if verbose else []) + ["-c", "-o", obj, os.path.join(CSRC, src)],
                                 stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
                for src, obj in zip(SOURCES, objects)]
        said = [job.communicate()[0] for job in jobs]
        if any(job.returncode != 0 for job in jobs):
            failed = "nvcc failed building libsparsecomm.so"
        if not failed:
            link = subprocess.run(flags + ["-shared", "-o", LIB] + objects, capture_output=True, text=True)
            said.append(link.stdout + link.stderr)
            if link.returncode != 0:
                failed = "nvcc failed linking libsparsecomm.so"
        if not failed and _calls_wanted():
            for command in _calls_commands():
                made = subprocess.run(command, capture_output=True, text=True)
                said.append(made.stdout + made.stderr)
                if made.returncode == 0:
                    break
            else:
                failed = f"the C++ compiler failed building {os.path.basename(CALLS)}"
    if failed or verbose:
        sys.stderr.write("".join(said))
    if failed:
        raise RuntimeError(failed)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
