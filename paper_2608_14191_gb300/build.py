"""Build the in-tree CUDA library ``libaatc.so`` for sm_103a with nvcc (no cmake).

Each translation unit compiles in parallel; the shared object lands next to this file, and with it
``_calls``, the Python extension through which the binding makes the paged calls (under the name that this
interpreter's modules have, so that another one does not load it).  The library needs no Python: where the
interpreter's headers are missing it is built alone.
"""
from __future__ import annotations

import concurrent.futures as cf
import os
import shutil
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libaatc.so")
CALLS = os.path.join(HERE, "_calls" + (sysconfig.get_config_var("EXT_SUFFIX") or ".so"))
SOURCES = ["planner.cpp", "planfile.cpp", "capi.cpp", "encode.cu", "decode.cu", "prefill.cu", "group.cu", "paged_api.cpp", "paged.cu",
           "selftest.cu"]
CALLS_SOURCE = "pycalls.cpp"
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found")


def _flags():
    return ARCH + ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC,-O2,-pthread",
                   "-I" + os.path.join(ROOT, "include"), "-I" + CSRC]


def _python_include() -> str | None:
    """The directory of the interpreter's headers, if they are installed."""
    path = sysconfig.get_paths()["include"]
    return path if os.path.exists(os.path.join(path, "Python.h")) else None


def _compile(src: str, verbose: bool) -> str:
    obj = os.path.join(BUILD, os.path.splitext(src)[0] + ".o")
    cmd = [_nvcc()] + _flags() + ["-c", os.path.join(CSRC, src), "-o", obj]
    if src == CALLS_SOURCE:
        cmd += ["-I" + _python_include()]
    if src.endswith(".cu") and verbose:
        cmd += ["-Xptxas", "-v"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"nvcc failed for {src}:\n{r.stdout}\n{r.stderr}")
    if verbose and (r.stdout or r.stderr):
        sys.stderr.write(r.stdout + r.stderr)
    return obj


def build(verbose: bool = False, force: bool = False) -> str:
    os.makedirs(BUILD, exist_ok=True)
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + [os.path.join(ROOT, "include", "aatc.h")]
    with_calls = _python_include() is not None
    built = [LIB] + ([CALLS] if with_calls else [])
    if not force and all(os.path.exists(p) for p in built):
        newest = max(os.path.getmtime(p) for p in deps)
        if min(os.path.getmtime(p) for p in built) >= newest:
            return LIB
    with cf.ThreadPoolExecutor(max_workers=len(SOURCES) + 1) as ex:
        calls = ex.submit(_compile, CALLS_SOURCE, verbose) if with_calls else None
        _link(LIB, list(ex.map(lambda s: _compile(s, verbose), SOURCES)) + ["-lpthread", "-ldl", "-lrt"])
        if calls is None:
            sys.stderr.write("Python's headers are missing: the extension of the paged calls is not built\n")
        else:
            _link(CALLS, [calls.result(), "-L" + HERE, "-l:" + os.path.basename(LIB), "-Xlinker", "-rpath,$ORIGIN"])
    return LIB


def _link(out: str, args):
    tmp = out + ".tmp"
    r = subprocess.run([_nvcc()] + ARCH + ["-shared", "-o", tmp] + args, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, out)


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv, force="-f" in sys.argv))
