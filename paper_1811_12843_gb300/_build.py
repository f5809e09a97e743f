"""Builds the engine's shared library (liblipz.so) for sm_103a with nvcc, in-tree, and the binding of
its operators to torch tensors (torch_operators.so) with the host compiler.

Each translation unit compiles in parallel; the work is skipped when a stamp of the sources
and flags is unchanged. Both go to ``paper_1811_12843_gb300/_lib/``.
"""

import concurrent.futures
import hashlib
import importlib.util
import os
import shutil
import subprocess
import sys
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
OUT_DIR = os.path.join(PKG, "_lib")
LIB = os.path.join(OUT_DIR, "liblipz.so")
BINDING = os.path.join(OUT_DIR, "torch_operators.so")

SOURCES = ["api.cu", "simt_kernels.cu", "gemm_tc.cu", "fwd_tc.cu", "bwd_tc.cu", "noalloc.cu",
           "conv_kernels.cu", "dcgan.cu", "conv_tc.cu", "operators.cu", "op_linear.cu", "op_gemm.cu",
           "op_norm.cu"]
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
FLAGS = ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC", "-Xcompiler", "-fvisibility=hidden",
         "--expt-relaxed-constexpr", "-I" + INCLUDE, "-I" + CSRC]


def _nvcc():
    for cand in (shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found")


def _torch_dir():
    """The installation of a torch with CUDA, found without importing it; None without one (and then no
    binding: the library is complete without it)."""
    spec = importlib.util.find_spec("torch")
    d = os.path.dirname(spec.origin) if spec is not None and spec.origin else None
    return d if d and os.path.exists(os.path.join(d, "lib", "libc10_cuda.so")) else None


def _cxx():
    for cand in (os.environ.get("CXX"), "g++", "c++"):
        if cand and shutil.which(cand):
            return cand
    raise RuntimeError("no host C++ compiler found")


def _run(cmd, what, verbose=False):
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("%s failed:\n%s\n%s" % (what, " ".join(cmd), r.stderr))
    if verbose and r.stderr:
        sys.stderr.write(r.stderr)


def _stamp():
    h = hashlib.sha256()
    # (the binding goes by torch's headers and Python's)
    torch_dir = _torch_dir()
    if torch_dir:
        with open(os.path.join(torch_dir, "version.py"), "rb") as f:
            h.update(f.read())
    h.update(sys.version.encode())
    for d in (CSRC, INCLUDE):
        for name in sorted(os.listdir(d)):
            p = os.path.join(d, name)
            if os.path.isfile(p):
                h.update(name.encode())
                with open(p, "rb") as f:
                    h.update(f.read())
    h.update(" ".join(ARCH + FLAGS).encode())
    h.update(os.uname().machine.encode())
    return h.hexdigest()


def build(force: bool = False, verbose: bool = False, extra_flags=()) -> str:
    """Compile and link the library if its sources changed; return the library path."""
    os.makedirs(OUT_DIR, exist_ok=True)
    stamp_file = os.path.join(OUT_DIR, "stamp")
    stamp = _stamp() + "|" + " ".join(extra_flags)
    built = os.path.exists(LIB) and (os.path.exists(BINDING) or not _torch_dir())
    if not force and built and os.path.exists(stamp_file):
        with open(stamp_file) as f:
            if f.read() == stamp:
                return LIB
    nvcc = _nvcc()
    obj_dir = os.path.join(OUT_DIR, "obj")
    os.makedirs(obj_dir, exist_ok=True)

    def compile_one(src):
        obj = os.path.join(obj_dir, src.replace(".cu", ".o"))
        cmd = [nvcc] + ARCH + FLAGS + list(extra_flags) + ["-c", os.path.join(CSRC, src), "-o", obj]
        _run(cmd, "nvcc of " + src, verbose)
        return obj

    torch_dir = _torch_dir()
    binding_obj = os.path.join(obj_dir, "torch_operators.o")

    def compile_binding():
        cuda = os.path.dirname(os.path.dirname(os.path.realpath(nvcc)))
        cmd = [_cxx(), "-O2", "-std=c++17", "-fPIC", "-fvisibility=hidden", "-I" + INCLUDE]
        for d in (os.path.join(torch_dir, "include"),
                  os.path.join(torch_dir, "include", "torch", "csrc", "api", "include"),
                  sysconfig.get_paths()["include"], os.path.join(cuda, "include")):
            cmd += ["-isystem", d]
        cmd += ["-c", os.path.join(CSRC, "torch_operators.cpp"), "-o", binding_obj]
        _run(cmd, "the binding's compilation", verbose)

    with concurrent.futures.ThreadPoolExecutor(max_workers=len(SOURCES) + 1) as ex:
        binding = ex.submit(compile_binding) if torch_dir else None
        objs = list(ex.map(compile_one, SOURCES))
        if binding:
            binding.result()
    tmp = LIB + ".tmp"
    _run([nvcc] + ARCH + ["-shared", "-o", tmp] + objs, "link")
    os.replace(tmp, LIB)
    if torch_dir:
        # (torch's libraries are loaded by then: the binding is imported after torch)
        tmp = BINDING + ".tmp"
        _run([_cxx(), "-shared", "-o", tmp, binding_obj, "-L" + OUT_DIR, "-llipz", "-Wl,-rpath,$ORIGIN",
              "-L" + os.path.join(torch_dir, "lib"), "-ltorch_python", "-ltorch", "-ltorch_cpu",
              "-lc10_cuda", "-lc10"], "the binding's link")
        os.replace(tmp, BINDING)
    with open(stamp_file, "w") as f:
        f.write(stamp)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose=True))
