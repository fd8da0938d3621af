"""Build the C-ABI shared library libfedoptima.so in-tree with nvcc for
sm_103a (GB300), and _binding.so, the compiled part of its Python binding, with
g++ against torch's headers.  Sources compile in parallel; objects go to _build/.
The library needs nvcc alone: without torch or g++ it is built and the binding
left out.

Several processes may call build() at once (one per rank under torchrun):
an exclusive file lock serialises them, and every object and the library
are written under a temporary name and renamed into place, so a process
never loads a half-written library."""
from __future__ import annotations

import concurrent.futures as cf
import fcntl
import importlib.util
import os
import shutil
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OUT = os.path.join(HERE, "libfedoptima.so")
BUILD = os.path.join(HERE, "_build")
BINDING = os.path.join(HERE, "_binding.so")

SOURCES = ["fo_server.cu", "k_elementwise.cu", "k_simt_conv.cu", "k_attention.cu", "k_tc_gemm.cu", "k_tc_gemm_fwd.cu", "k_tc_gemm_dgrad.cu", "k_tc_gemm_wgrad.cu", "k_head.cu", "k_vec.cu", "fo_noalloc.cu", "k_attention_tc.cu", "fo_preproc.cu", "k_mobile.cu", "k_scored.cu", "k_scored_fwd.cu", "k_scored_bwd.cu", "k_dropout.cu", "k_embedding.cu", "k_norm.cu", "k_orthogonalize.cu"]
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
FLAGS = ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC", "--expt-relaxed-constexpr",
         "-Xcompiler", "-fvisibility=hidden"]


def nvcc():
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found")


def _torch():
    """torch's folder, without importing it, or None."""
    spec = importlib.util.find_spec("torch")
    return spec.submodule_search_locations[0] if spec else None


def _without_binding():
    """Why the binding cannot be built here, or None."""
    root = _torch()
    if root is None:
        return "torch is not installed"
    if not os.path.exists(os.path.join(root, "include", "torch", "csrc", "autograd", "python_variable.h")):
        return "torch has no headers here"
    return None if shutil.which("g++") else "g++ was not found"


def _run(cmd, what, tmp):
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        if os.path.exists(tmp):
            os.remove(tmp)
        raise RuntimeError(f"{what}:\n{r.stdout}\n{r.stderr}")
    return r.stderr


def _made_for():
    """What the binding's binary interface goes by: this Python, and torch's folder, version and revision."""
    root = _torch()
    with open(os.path.join(root, "version.py")) as f:
        return f"{sys.version}\n{root}\n{f.read()}"


def _binding_files():
    return os.path.join(BUILD, "fo_binding.o"), os.path.join(CSRC, "fo_binding.cpp")


def _is_current():
    """Whether the binding's object is of its source and for this torch."""
    obj, src = _binding_files()
    try:
        with open(obj + ".txt") as f:
            if f.read() != _made_for():
                return False
        deps = [src, os.path.join(HERE, "..", "include", "fedoptima.h")]
        return all(os.path.getmtime(obj) >= os.path.getmtime(d) for d in deps)
    except (OSError, TypeError):               # no object, or no torch
        return False


def _compile_binding():
    obj, src = _binding_files()
    if _is_current():
        return obj, ""
    include = os.path.join(_torch(), "include")
    cuda = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(nvcc()))), "include")
    tmp = f"{obj}.{os.getpid()}.tmp"
    log = _run(["g++", "-O2", "-std=c++17", "-fPIC", "-fvisibility=hidden", "-I" + sysconfig.get_paths()["include"], "-isystem", include,
                "-isystem", os.path.join(include, "torch", "csrc", "api", "include"), "-isystem", cuda, "-c", src, "-o", tmp],
               "g++ failed for fo_binding.cpp", tmp)
    os.replace(tmp, obj)
    with open(obj + ".txt", "w") as f:        # last: without it the object is made again
        f.write(_made_for())
    return obj, log


def _link_binding(obj):
    if os.path.exists(BINDING) and os.path.getmtime(BINDING) >= max(os.path.getmtime(obj), os.path.getmtime(OUT)):
        return
    tmp = f"{BINDING}.{os.getpid()}.tmp"
    _run(["g++", "-shared", "-o", tmp, obj, "-L" + HERE, "-l:" + os.path.basename(OUT), "-Wl,-rpath,$ORIGIN", "-L" + os.path.join(_torch(), "lib"),
          "-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_cuda", "-ltorch_python"], "link of _binding.so failed", tmp)
    os.replace(tmp, BINDING)


def _compile(src, extra):
    obj = os.path.join(BUILD, os.path.splitext(src)[0] + ".o")
    srcp = os.path.join(CSRC, src)
    deps = [srcp] + [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".h", ".hpp", ".cuh"))]
    deps.append(os.path.join(HERE, "..", "include", "fedoptima.h"))
    if os.path.exists(obj) and all(os.path.getmtime(obj) >= os.path.getmtime(d) for d in deps):
        return obj, ""
    tmp = f"{obj}.{os.getpid()}.tmp"
    log = _run([nvcc(), *ARCH, *FLAGS, *extra, "-c", srcp, "-o", tmp], f"nvcc failed for {src}", tmp)
    os.replace(tmp, obj)
    return obj, log


def build(verbose=False, extra=()):
    os.makedirs(BUILD, exist_ok=True)
    with open(os.path.join(BUILD, ".lock"), "w") as lock:
        try:
            fcntl.flock(lock, fcntl.LOCK_EX)  # released when the file closes
        except OSError:                       # a filesystem without locks: build unserialised
            pass
        with cf.ThreadPoolExecutor(max_workers=min(len(SOURCES), os.cpu_count() or 4)) as ex:
            why = _without_binding()
            binding = None if why else ex.submit(_compile_binding)
            results = list(ex.map(lambda s: _compile(s, list(extra)), SOURCES))
        objs = [o for o, _ in results]
        if verbose:
            for _, log in results:
                if log:
                    sys.stderr.write(log)
        newest = max(os.path.getmtime(o) for o in objs)
        if not os.path.exists(OUT) or os.path.getmtime(OUT) < newest:
            tmp = f"{OUT}.{os.getpid()}.tmp"
            _run([nvcc(), *ARCH, "-shared", "-o", tmp, *objs], "link failed", tmp)
            os.replace(tmp, OUT)
        if binding is None:
            if os.path.exists(BINDING) and not _is_current():
                os.remove(BINDING)             # made for another torch, or from another source
            sys.stderr.write(f"_binding.so is left out ({why}): embedding, norms and orthogonalised updates have no Python entry points\n")
        else:
            obj, log = binding.result()
            if verbose and log:
                sys.stderr.write(log)
            _link_binding(obj)
    return OUT


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv, extra=[a for a in sys.argv[1:] if a != "-v"]))
