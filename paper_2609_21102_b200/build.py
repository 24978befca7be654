"""Builds the CUDA library in-tree, paper_2609_21102_b200/libdeflpolar.so (sm_100a only), and the Python module over it."""
import os
import shutil
import subprocess
import sys
import warnings

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libdeflpolar.so")
NATIVE = os.path.join(HERE, "_native.so")
SOURCES = ["api.cu", "psd.cu", "gemm_simt.cu", "gemm_tc.cu", "panel.cu", "optim.cu", "mx4.cu", "mx4_gemm.cu"]
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC", "--use_fast_math=false"]


def _stale(target, deps):
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(d) > t for d in deps)


def build(force=False, verbose=False):
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    headers = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".cuh", ".h"))]
    headers.append(os.path.join(os.path.dirname(HERE), "include", "defl.h"))
    objs = []
    procs = []
    for src in SOURCES:
        s = os.path.join(CSRC, src)
        if not os.path.exists(s):
            continue
        o = os.path.join(CSRC, src.replace(".cu", ".o"))
        objs.append(o)
        if force or _stale(o, [s] + headers):
            cmd = [nvcc] + [f for f in NVCC_FLAGS if not f.startswith("--use_fast_math")] + ["-c", s, "-o", o]
            if verbose:
                cmd.insert(1, "-Xptxas")
                cmd.insert(2, "-v")
            procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    failed = False
    for src, p in procs:
        out, _ = p.communicate()
        if p.returncode != 0 or verbose:
            sys.stderr.write("[%s]\n%s\n" % (src, out))
        failed |= p.returncode != 0
    if failed:
        raise RuntimeError("nvcc failed")
    if force or procs or _stale(LIB, objs):
        cmd = [nvcc, "-shared", "-o", LIB] + objs + ["-gencode", "arch=compute_100a,code=sm_100a", "-lcudart"]
        subprocess.run(cmd, check=True)
    build_native(force)
    return LIB


def build_native(force=False):
    """The Python module that calls the library without ctypes (csrc/native.cpp), against the installed torch's headers. Its ABI is that of
    the torch and the Python it was built with, whose versions stand beside it. Where a compiler or headers are missing the library
    serves without it: a warning here, an ImportError from the calls that need it."""
    import sysconfig
    import torch
    src, built_with = os.path.join(CSRC, "native.cpp"), NATIVE + ".versions"
    versions = "torch %s, python %s\n" % (torch.__version__, sys.version)
    same = os.path.exists(built_with) and open(built_with).read() == versions
    if same and not (force or _stale(NATIVE, [src, os.path.join(os.path.dirname(HERE), "include", "defl.h")])):
        return NATIVE
    for old in (NATIVE, built_with):
        if os.path.exists(old):
            os.remove(old)
    root, python = os.path.dirname(torch.__file__), sysconfig.get_paths()["include"]
    missing = [x for x in (os.path.join(python, "Python.h"), os.path.join(root, "include", "torch", "csrc", "autograd", "python_variable.h"))
               if not os.path.exists(x)] + ([] if shutil.which("g++") else ["g++"])
    if missing:
        warnings.warn("%s not built, AdamW, the gradient norm and the 4-bit operators cannot be called from Python: no %s"
                      % (os.path.basename(NATIVE), ", ".join(missing)))
        return None
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-w", "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch._C._GLIBCXX_USE_CXX11_ABI,
           "-I" + os.path.join(root, "include"), "-I" + os.path.join(root, "include", "torch", "csrc", "api", "include"),
           "-I" + python, "-I/usr/local/cuda/include", src, "-o", NATIVE,
           # torch's libraries are in the process already; the library is found beside the module
           "-L" + os.path.join(root, "lib"), "-ltorch_python", "-ltorch_cpu", "-ltorch_cuda", "-lc10", "-lc10_cuda",
           "-L" + HERE, "-l:libdeflpolar.so", "-Wl,-rpath,$ORIGIN"]
    subprocess.run(cmd, check=True)
    with open(built_with, "w") as f:
        f.write(versions)
    return NATIVE


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
