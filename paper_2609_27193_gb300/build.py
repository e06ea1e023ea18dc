"""Builds liblayercheck.so in-tree for sm_103a with nvcc (no cmake).

Each .cu under csrc/ is compiled in parallel to an object under _build/,
then linked into paper_2609_27193_gb300/liblayercheck.so with the CUDA
runtime linked statically.  Only the lc_* entry points are exported.

The operators' binding over torch tensors (binding/ops_binding.cpp) becomes the
extension module _ops.so beside it, with g++ and torch's headers, at the same
time.  Without torch there is none: the library and its C ABI need neither.
"""
import concurrent.futures as cf
import importlib.metadata
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
BUILD = os.path.join(ROOT, "_build")
LIB = os.path.join(PKG, "liblayercheck.so")
BINDING = os.path.join(PKG, "binding", "ops_binding.cpp")
BINDING_LIB = os.path.join(PKG, "_ops.so")
BINDING_STAMP = os.path.join(BUILD, "ops_binding.for")

ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
NVFLAGS = ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC,-ffp-contract=off",
           "-Xptxas", "-warn-spills", "--expt-relaxed-constexpr", "-I", INCLUDE, "-I", CSRC]


def _nvcc():
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found: liblayercheck.so cannot be built")


def _sources():
    return sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".cu"))


def _inputs():
    files = _sources() + [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".cuh")]
    return files + [os.path.join(INCLUDE, "layercheck.h"), os.path.abspath(__file__)]


def up_to_date():
    if not os.path.exists(LIB):
        return False
    t = os.path.getmtime(LIB)
    return all(os.path.getmtime(f) <= t for f in _inputs())


def binding_for():
    """What the binding is compiled against: the torch and the Python found here; None without torch."""
    spec = importlib.util.find_spec("torch")
    if spec is None:
        return None
    try:
        version = importlib.metadata.version("torch")
    except importlib.metadata.PackageNotFoundError:
        version = "?"
    return "torch %s at %s, %s" % (version, spec.origin, sysconfig.get_config_var("SOABI"))


def binding_up_to_date():
    if not os.path.exists(BINDING_STAMP) or open(BINDING_STAMP).read() != binding_for():
        return False
    inputs = [BINDING, os.path.join(INCLUDE, "layercheck.h"), os.path.abspath(__file__)]
    return os.path.exists(BINDING_LIB) and all(os.path.getmtime(f) <= os.path.getmtime(BINDING_LIB) for f in inputs)


def compile_binding():
    """ops_binding.cpp to an object; returns it and torch's library folder."""
    import torch
    home = os.path.dirname(torch.__file__)
    include = [os.path.join(home, "include"), os.path.join(home, "include", "torch", "csrc", "api", "include"),
               sysconfig.get_paths()["include"], os.path.join(os.path.dirname(os.path.dirname(_nvcc())), "include"),
               INCLUDE]
    os.makedirs(BUILD, exist_ok=True)
    obj = os.path.join(BUILD, "ops_binding.o")
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-fvisibility=hidden",
           "-D_GLIBCXX_USE_CXX11_ABI=%d" % int(torch._C._GLIBCXX_USE_CXX11_ABI),
           *[x for d in include for x in ("-isystem" if d != INCLUDE else "-I", d)], "-c", BINDING, "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("g++ failed on %s:\n%s%s" % (BINDING, r.stdout, r.stderr[-4000:]))
    return obj, os.path.join(home, "lib")


def link_binding(obj, torch_lib):
    tmp = BINDING_LIB + ".tmp%d" % os.getpid()
    cmd = ["g++", "-shared", "-o", tmp, obj, "-L", PKG, "-l:liblayercheck.so", "-L", torch_lib, "-ltorch_python",
           "-ltorch_cpu", "-ltorch_cuda", "-lc10_cuda", "-lc10", "-Wl,-rpath,$ORIGIN"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed:\n%s%s" % (r.stdout, r.stderr))
    os.replace(tmp, BINDING_LIB)
    with open(BINDING_STAMP, "w") as fh:
        fh.write(binding_for())


def build(force=False, verbose=False, extra_flags=()):
    """Compile and link; returns the library path."""
    with cf.ThreadPoolExecutor(max_workers=1) as ex:
        wanted = binding_for() is not None and (force or not binding_up_to_date())
        binding = ex.submit(compile_binding) if wanted else None
        lib = build_library(force, verbose, extra_flags)
        if binding is not None:
            link_binding(*binding.result())
    return lib


def build_library(force=False, verbose=False, extra_flags=()):
    if not force and up_to_date():
        return LIB
    nvcc = _nvcc()
    os.makedirs(BUILD, exist_ok=True)
    srcs = _sources()

    def compile_one(src):
        obj = os.path.join(BUILD, os.path.basename(src)[:-3] + ".o")
        cmd = [nvcc, *ARCH, *NVFLAGS, *extra_flags, "-c", src, "-o", obj]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError("nvcc failed on %s:\n%s%s" % (src, r.stdout, r.stderr))
        return obj, r.stdout + r.stderr

    with cf.ThreadPoolExecutor(max_workers=min(8, len(srcs))) as ex:
        results = list(ex.map(compile_one, srcs))
    if verbose:
        for obj, log in results:
            if log.strip():
                print(log)
    vscript = os.path.join(BUILD, "exports.map")
    with open(vscript, "w") as fh:
        fh.write("{ global: lc_*; local: *; };\n")
    tmp = LIB + ".tmp%d" % os.getpid()
    cmd = [nvcc, *ARCH, "-shared", "-o", tmp, *[o for o, _ in results], "-Xlinker", "--soname=liblayercheck.so",
           "-Xlinker", "--version-script=" + vscript, "-cudart", "static"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed:\n%s%s" % (r.stdout, r.stderr))
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
