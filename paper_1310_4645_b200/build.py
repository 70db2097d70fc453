"""Builds librd.so (CUDA kernels + C ABI) in-tree with nvcc for sm_100a, and _rd_torch.so (tensor marshalling) beside it.

librd.so needs no torch; where there is none, or one without CUDA, it is all that is built.
"""
from __future__ import annotations

import importlib.util
import os
import re
import shutil
import subprocess
import sys
import sysconfig
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "librd.so")
TORCH_LIB = os.path.join(HERE, "_rd_torch.so")
SOURCES = ["rd_api.cpp", "rd_sched.cpp", "rd_compile.cpp", "rd_kernels.cu", "rd_faithful.cu", "rd_broadcast.cu",
           "rd_vocab_api.cpp", "rd_embed.cu", "rd_vocab.cu", "rd_block_api.cpp", "rd_norm.cu", "rd_norm_f32.cu", "rd_norm_bf16.cu", "rd_norm_fp16.cu",
           "rd_gated.cu"]
HEADERS = ["rd_internal.h", "rd_kernels.h", "rd_checks.h", "rd_vocab.h", "rd_block.h", "rd_norm_rows.h", "rd_norm_shape.h",
           "rd_norm_kernels.h", "rd_mma.h", "rd_launch.h", "rd_ptx.h", "rd_ring.h"]
# rd_kernels.cu is compiled once per element type (-DRD_DT=k: that type's kernels; the 16-bit types count
# twice, once for sum and product and once for max and min) and once without (launch shapes and dispatch),
# side by side
KERNEL_DTYPES = 8
NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-Xcompiler", "-fPIC,-Wall,-Wextra,-fvisibility=hidden",
]
LINK_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-shared", "-cudart", "static"]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", "nvcc"):
        if cand and (os.path.isabs(cand) and os.path.exists(cand) or not os.path.isabs(cand)):
            return cand
    return "nvcc"


def _torch_dir() -> str | None:
    """The installed torch's folder (found, not imported); None where there is none, or one without CUDA."""
    spec = importlib.util.find_spec("torch")
    for place in (spec and spec.submodule_search_locations) or ():
        if os.path.exists(os.path.join(place, "lib", "libc10_cuda.so")):
            return place
    return None


def _torch_built_for(torch_dir: str) -> str:
    """What the tensor module depends on besides its sources: it uses torch's and the interpreter's C++ and C interfaces."""
    with open(os.path.join(torch_dir, "version.py")) as f:
        version = re.search(r"^__version__\s*=\s*['\"](.+?)['\"]", f.read(), re.M)
    return "torch %s, %s\n" % (version.group(1) if version else "", sys.implementation.cache_tag)


def _torch_stamp() -> str:
    """The file that says what the tensor module was built for."""
    return os.path.join(os.path.dirname(TORCH_LIB), "_build", "rd_torch.txt")


def _stamped() -> str:
    try:
        with open(_torch_stamp()) as f:
            return f.read()
    except FileNotFoundError:
        return ""


def stale() -> bool:
    libraries, sources = [LIB], SOURCES + HEADERS
    torch_dir = _torch_dir()
    if torch_dir:
        if _stamped() != _torch_built_for(torch_dir):
            return True
        libraries, sources = libraries + [TORCH_LIB], sources + ["rd_torch.cpp"]
    if not all(map(os.path.exists, libraries)):
        return True
    built = min(map(os.path.getmtime, libraries))
    deps = [os.path.join(CSRC, f) for f in sources] + [os.path.join(ROOT, "include", "rd.h")]
    return any(os.path.getmtime(d) > built for d in deps)


def _torch_module(work: str, torch_dir: str) -> str:
    """Compiles the marshalling module against the installed torch; it is linked to librd.so beside it."""
    cuda = os.path.dirname(os.path.dirname(_nvcc())) if os.path.isabs(_nvcc()) else "/usr/local/cuda"
    obj = os.path.join(work, "rd_torch.o")
    subprocess.check_call(["g++", "-O2", "-std=c++17", "-fPIC", "-fvisibility=hidden", "-Wall", "-Wextra", "-c", "-o", obj,
                           os.path.join(CSRC, "rd_torch.cpp"), "-I", os.path.join(ROOT, "include"),
                           "-isystem", os.path.join(torch_dir, "include"), "-isystem", os.path.join(torch_dir, "include", "torch", "csrc", "api", "include"),
                           "-isystem", sysconfig.get_paths()["include"], "-isystem", os.path.join(cuda, "include")])
    return obj


def _link_torch_module(obj: str, torch_dir: str) -> None:
    tmp = TORCH_LIB + ".%d.tmp" % os.getpid()
    subprocess.check_call(["g++", "-shared", "-o", tmp, obj, "-L", os.path.join(torch_dir, "lib"), "-ltorch_python", "-ltorch_cuda", "-ltorch_cpu",
                           "-lc10_cuda", "-lc10", "-L", HERE, "-l:" + os.path.basename(LIB), "-Wl,-rpath,$ORIGIN"])
    os.replace(tmp, TORCH_LIB)
    os.makedirs(os.path.dirname(_torch_stamp()), exist_ok=True)
    with open(_torch_stamp(), "w") as f:
        f.write(_torch_built_for(torch_dir))


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile when sources are newer than the library.  Returns the library path."""
    if not force and not stale():
        return LIB
    nvcc = _nvcc()
    common = [nvcc, *NVCC_FLAGS, "-I", os.path.join(ROOT, "include"), "-I", CSRC]
    if verbose:
        common += ["-Xptxas", "-v"]
    work = tempfile.mkdtemp(prefix="librd_build_")
    try:
        units = []                                   # (object file, source, extra flags)
        for f in SOURCES:
            stem = os.path.splitext(f)[0]
            units.append((os.path.join(work, stem + ".o"), f, []))
            if f == "rd_kernels.cu":
                # (a unit that serves one element type leaves the other types' helpers unreferenced: diagnostic 177)
                units[-1] = (units[-1][0], f, ["-diag-suppress", "177"])
                for k in range(KERNEL_DTYPES):
                    units.append((os.path.join(work, "%s_dt%d.o" % (stem, k)), f, ["-DRD_DT=%d" % k, "-diag-suppress", "177"]))

        def compile_one(unit):
            obj, src, extra = unit
            subprocess.check_call(common + extra + ["-c", "-o", obj, os.path.join(CSRC, src)])
            return obj

        with ThreadPoolExecutor(max_workers=min(len(units) + 1, os.cpu_count() or 4)) as pool:
            torch_dir = _torch_dir()
            marshalling = pool.submit(_torch_module, work, torch_dir) if torch_dir else None
            objs = list(pool.map(compile_one, units))
        tmp = LIB + ".%d.tmp" % os.getpid()
        subprocess.check_call([nvcc, *LINK_FLAGS, "-o", tmp] + objs)
        os.replace(tmp, LIB)
        if marshalling:
            _link_torch_module(marshalling.result(), torch_dir)
    finally:
        shutil.rmtree(work, ignore_errors=True)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
