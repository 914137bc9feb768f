"""Build libdas.so (the CUDA library behind include/das.h) in place for sm_103a,
and _calls.so (the Python binding's module in C++, against PyTorch's headers).

    python paper_2609_34538_gb300/build.py

Each .cu under csrc/ is compiled in parallel with nvcc, then linked into
paper_2609_34538_gb300/libdas.so.  A rebuild happens only when a source or
header is newer than the libraries.
"""
import concurrent.futures as cf
import importlib.util
import os
import subprocess
import sys
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
OUT_DIR = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libdas.so")
CALLS_SRC = os.path.join(CSRC, "calls.cpp")
CALLS = os.path.join(PKG, "_calls.so")
NVCC = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
FLAGS = ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC", "-I", INCLUDE, "-I", CSRC]


def _sources():
    return sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".cu"))


def _inputs():
    hdrs = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".h")]
    hdrs += [os.path.join(INCLUDE, f) for f in os.listdir(INCLUDE) if f.endswith(".h")]
    torch = os.path.join(_torch_dir(), "version.py")  # _calls.so is for the PyTorch it was built with
    return _sources() + hdrs + [CALLS_SRC, torch, os.path.abspath(__file__)]


def up_to_date():
    if not (os.path.exists(LIB) and os.path.exists(CALLS)):
        return False
    t = min(os.path.getmtime(LIB), os.path.getmtime(CALLS))
    return all(os.path.getmtime(f) <= t for f in _inputs())


def _compile(src, extra):
    obj = os.path.join(OUT_DIR, os.path.basename(src)[:-3] + ".o")
    cmd = [NVCC, *ARCH, *FLAGS, *extra, "-c", src, "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"nvcc failed on {src}:\n{r.stdout}\n{r.stderr}")
    return obj, r.stderr


def _run(cmd, what):
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"{what} failed:\n{r.stdout}\n{r.stderr}")


def _torch_dir():  # (without importing it, which takes longer than the compilation)
    return importlib.util.find_spec("torch").submodule_search_locations[0]


def _compile_calls():
    obj = os.path.join(OUT_DIR, "calls.o")
    torch, cuda = os.path.join(_torch_dir(), "include"), os.path.dirname(os.path.dirname(NVCC))
    dirs = [INCLUDE, torch, os.path.join(torch, "torch", "csrc", "api", "include"),
            os.path.join(cuda, "include"), sysconfig.get_paths()["include"]]
    _run(["g++", "-O2", "-std=c++17", "-fPIC", "-fvisibility=hidden", *(f"-I{d}" for d in dirs),
          "-c", CALLS_SRC, "-o", obj], f"g++ on {CALLS_SRC}")
    return obj


def _link_calls(obj):
    """Against libdas.so beside it, and the libraries that `import torch` has loaded."""
    tmp = CALLS + ".tmp"
    _run(["g++", "-shared", "-o", tmp, obj, f"-L{PKG}", "-l:libdas.so", "-Wl,-rpath,$ORIGIN",
          f"-L{os.path.join(_torch_dir(), 'lib')}", "-ltorch_python", "-ltorch_cpu", "-lc10_cuda",
          "-lc10"], "linking _calls.so")
    os.replace(tmp, CALLS)


def build(force=False, verbose=False):
    if not force and up_to_date():
        return LIB
    os.makedirs(OUT_DIR, exist_ok=True)
    extra = ["-Xptxas", "-v"] if verbose else []
    with cf.ThreadPoolExecutor(max_workers=len(_sources()) + 1) as ex:
        calls = ex.submit(_compile_calls)
        results = list(ex.map(lambda s: _compile(s, extra), _sources()))
    if verbose:
        for _, log in results:
            sys.stderr.write(log)
    tmp = LIB + ".tmp"
    cmd = [NVCC, *ARCH, "-shared", "-o", tmp] + [o for o, _ in results]
    _run(cmd, "link")
    os.replace(tmp, LIB)
    _link_calls(calls.result())  # (last: libdas.so does not need it)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
