"""Build ``libbmlp.so`` (the CUDA library behind include/bmlp.h) with nvcc.

One ``-gencode arch=compute_103a,code=sm_103a`` target; the translation units
are compiled in parallel and linked with the static CUDA runtime, so the
library needs only the driver at run time.
"""
from __future__ import annotations

import concurrent.futures as cf
import importlib.util
import os
import runpy
import shutil
import subprocess
import sysconfig
import threading

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
ROOT = os.path.dirname(HERE)
LIB = os.path.join(HERE, "libbmlp.so")
SOURCES = ["bmlp_api.cu", "bmlp_noalloc.cu", "kern_forward.cu", "kern_forward_tc.cu", "kern_eval_tc.cu",
           "kern_update.cu", "kern_binarize.cu", "kern_expand.cu", "kern_peaks.cu", "kern_forward_b1.cu",
           "kern_update_rows.cu", "kern_update_ws.cu", "kern_quantize.cu", "kern_int8.cu",
           "kern_int8_few.cu", "kern_int8_tile.cu", "kern_int8_pair.cu", "kern_mx4_quantize.cu",
           "kern_mx4_tile.cu", "kern_mx4_pair.cu"]
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
FLAGS = ["-O3", "-std=c++17", "-lineinfo", "-Xcompiler", "-fPIC,-ffp-contract=off",
         "--expt-relaxed-constexpr", "-I", os.path.join(ROOT, "include")]


def nvcc() -> str:
    for cand in (os.environ.get("NVCC"), "/usr/local/cuda/bin/nvcc", shutil.which("nvcc")):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found")


def _stale(out: str, deps) -> bool:
    if not os.path.exists(out):
        return True
    t = os.path.getmtime(out)
    return any(os.path.getmtime(d) > t for d in deps)


def marshal_path(version: str, git_version: str) -> str:
    """The marshalling of torch tensors (csrc/marshal.cpp) for this interpreter and that torch, whose tensors it
    reads as they lie in memory: under a name of its own for each, so that no other one's is ever loaded."""
    tag = "".join(c if c.isalnum() or c in ".+" else "_" for c in "%s-%s" % (version, (git_version or "")[:12]))
    return os.path.join(HERE, "_marshal-%s.%s.so" % (tag, sysconfig.get_config_var("SOABI")))


def _marshal_job(force: bool):
    """The compiler's command for the marshalling of torch tensors, None where it is up to date or
    there is no torch to build it with."""
    src = os.path.join(CSRC, "marshal.cpp")
    try:
        found = importlib.util.find_spec("torch")
    except (ImportError, ValueError):
        found = None
    if found is None or not found.origin:
        return None
    at = os.path.dirname(found.origin)
    header = os.path.join(at, "include", "torch", "csrc", "autograd", "python_variable.h")
    if not os.path.exists(header):
        return None
    torch = runpy.run_path(os.path.join(at, "version.py"))    # (assignments alone)
    out = marshal_path(torch["__version__"], torch.get("git_version"))
    if not (force or _stale(out, [src, os.path.join(ROOT, "include", "bmlp.h"), os.path.join(at, "version.py")])):
        return None
    cuda = os.path.join(os.path.dirname(os.path.dirname(nvcc())), "include")
    return [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-shared", "-fPIC", "-I", os.path.join(ROOT, "include"),
            "-I", os.path.join(at, "include"), "-I", os.path.join(at, "include", "torch", "csrc", "api", "include"),
            "-I", sysconfig.get_paths()["include"], "-I", cuda, src, "-L", os.path.join(at, "lib"),
            "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda", "-o", out]


def _make_marshal(cmd) -> None:
    """An accelerator of the binding alone: without it the calls go the interpreter's way."""
    out = cmd[-1] + ".tmp%d" % os.getpid()
    res = subprocess.run(cmd[:-1] + [out], capture_output=True, text=True)
    if res.returncode == 0:
        os.replace(out, cmd[-1])
    else:
        print("csrc/marshal.cpp is not built; calls with torch tensors take some 4 us longer:\n" + res.stderr[-2000:])


def build(force: bool = False, verbose: bool = False, extra=()) -> str:
    objdir = os.path.join(HERE, "_build")
    os.makedirs(objdir, exist_ok=True)
    headers = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".cuh")]
    headers.append(os.path.join(ROOT, "include", "bmlp.h"))
    objs, jobs = [], []
    marshal = _marshal_job(force)
    beside = threading.Thread(target=_make_marshal, args=(marshal,)) if marshal else None
    if beside:
        beside.start()
    for src in SOURCES:
        sp = os.path.join(CSRC, src)
        op = os.path.join(objdir, src.replace(".cu", ".o"))
        objs.append(op)
        if force or _stale(op, [sp] + headers):
            jobs.append([nvcc(), *ARCH, *FLAGS, *extra, "-c", sp, "-o", op])
    if jobs:
        with cf.ThreadPoolExecutor(max_workers=len(jobs)) as ex:
            for cmd, res in zip(jobs, ex.map(lambda c: subprocess.run(c, capture_output=True, text=True), jobs)):
                if verbose or res.returncode != 0:
                    print(" ".join(cmd))
                    print(res.stdout + res.stderr)
                if res.returncode != 0:
                    raise RuntimeError("nvcc failed on " + cmd[-3])
    if force or jobs or _stale(LIB, objs):
        tmp = LIB + ".tmp%d" % os.getpid()
        cmd = [nvcc(), *ARCH, "-shared", "-cudart", "static", "-o", tmp, *objs]
        res = subprocess.run(cmd, capture_output=True, text=True)
        if res.returncode != 0:
            print(" ".join(cmd))
            print(res.stdout + res.stderr)
            raise RuntimeError("link failed")
        os.replace(tmp, LIB)
    if beside:
        beside.join()
    return LIB


if __name__ == "__main__":
    import sys
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
