"""Builds libmlkv_gb300.so in-tree with nvcc for sm_103a.

Each .cu is compiled in parallel to an object, then linked into one shared
library that exports the C ABI of include/mlkv_gpu.h and include/mlkv_dense.h.
No fast-math: every floating-point operation of the store's kernels is an
explicitly rounded intrinsic, and --fmad=false keeps the compiler from
contracting any other.  The dense operators are held to a tolerance, not to an
order of operations, and may contract.

Beside it _dense_calls.so, by g++: the dense operators' calls from Python
(csrc/dense_calls.cpp), against the installed torch, and built anew with another
torch.  Where that cannot be built (no headers of Python's or torch's), the
library is there all the same, and dense.py makes the calls by ctypes.
"""
import concurrent.futures as cf
import importlib.metadata
import importlib.util
import os
import shutil
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
ROOT = os.path.dirname(HERE)
LIB = os.path.join(HERE, "libmlkv_gb300.so")
CALLS = os.path.join(HERE, "_dense_calls.so")
BUILD = os.path.join(ROOT, "_build")
CALLS_SOURCE = "dense_calls.cpp"
HEADERS = [os.path.join(ROOT, "include", f) for f in ("mlkv_gpu.h", "mlkv_dense.h")]
SOURCES = ["mlkv_index.cu", "mlkv_sort.cu", "mlkv_apply.cu", "mlkv_plan.cu", "mlkv_table.cu", "mlkv_tier.cu", "mlkv_static.cu"]
DENSE = ["dense_norm.cu", "dense_norm_backward.cu", "dense_linear.cu", "dense_gated.cu", "dense_xent.cu",
         "dense_logprobs.cu", "dense_adamw.cu"]
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
FLAGS = ["-O3", "-std=c++17", "-lineinfo", "-Xcompiler", "-fPIC",
         "-Xcompiler", "-ffp-contract=off", f"-I{os.path.join(ROOT, 'include')}"]


def nvcc() -> str:
    for cand in (shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found")


def _newer(out: str, sources) -> bool:
    """Whether `out` is there and no older than what it is made of."""
    if not os.path.exists(out):
        return False
    t = os.path.getmtime(out)
    return all(os.path.getmtime(f) <= t for f in [*sources, *HEADERS, os.path.abspath(__file__)])


def _torch_version() -> str:
    try:
        return importlib.metadata.version("torch")
    except importlib.metadata.PackageNotFoundError:
        return ""


def _calls_torch() -> str:
    """The file with the version of torch that the extension module was built against."""
    return os.path.join(BUILD, "dense_calls.torch")


def library_up_to_date() -> bool:
    return _newer(LIB, [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".cu", ".cuh"))])


def calls_up_to_date() -> bool:
    if not _newer(CALLS, [os.path.join(CSRC, CALLS_SOURCE)]) or not os.path.exists(_calls_torch()):
        return False
    with open(_calls_torch()) as f:
        return f.read() == _torch_version()


def up_to_date() -> bool:
    return library_up_to_date() and calls_up_to_date()


def build_calls() -> str:
    """The extension module of the dense operators' calls."""
    spec = importlib.util.find_spec("torch")
    if spec is None:
        raise RuntimeError("torch is not installed")
    torch = spec.submodule_search_locations[0]
    cuda = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(nvcc()))), "include")
    include = [os.path.join(ROOT, "include"), sysconfig.get_paths()["include"], os.path.join(torch, "include"),
               os.path.join(torch, "include", "torch", "csrc", "api", "include"), cuda]
    tmp = CALLS + f".tmp{os.getpid()}"
    cmd = [shutil.which("g++") or "g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-fvisibility=hidden", *(f"-I{d}" for d in include),
           os.path.join(CSRC, CALLS_SOURCE), "-o", tmp, f"-L{os.path.join(torch, 'lib')}",
           *(f"-l{n}" for n in ("torch_python", "torch", "torch_cpu", "torch_cuda", "c10", "c10_cuda"))]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"g++ failed on {CALLS_SOURCE}:\n{r.stderr}")
    os.replace(tmp, CALLS)
    with open(_calls_torch(), "w") as f:
        f.write(_torch_version())
    return CALLS


def build(force: bool = False, verbose: bool = False, extra=()) -> str:
    # MLKV_NVCC_FLAGS: extra nvcc flags, e.g. -D overrides of the kernels'
    # tuning constants for a sweep; a build with them is always forced.
    env_extra = os.environ.get("MLKV_NVCC_FLAGS", "").split()
    extra = [*extra, *env_extra]
    library = force or bool(env_extra) or not library_up_to_date()
    calls = force or not calls_up_to_date()
    if not library and not calls:
        return LIB
    os.makedirs(BUILD, exist_ok=True)
    with cf.ThreadPoolExecutor(max_workers=1) as ex:
        module = ex.submit(build_calls) if calls else None
        if library:
            build_library(verbose, extra)
        try:
            if module:
                module.result()
        except (RuntimeError, OSError) as e:
            if os.path.exists(CALLS):  # (of other sources, or another torch)
                os.remove(CALLS)
            sys.stderr.write(f"{os.path.basename(CALLS)} cannot be built, the dense operators are called by ctypes: {e}\n")
    return LIB


def build_library(verbose: bool = False, extra=()) -> str:
    cc = nvcc()

    def compile_one(src):
        obj = os.path.join(BUILD, src.replace(".cu", ".o"))
        exact = [] if src in DENSE else ["--fmad=false"]
        cmd = [cc, *ARCH, *FLAGS, *exact, *extra, "-c", os.path.join(CSRC, src), "-o", obj]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"nvcc failed on {src}:\n{r.stderr}")
        if verbose and r.stderr:
            sys.stderr.write(r.stderr)
        return obj

    with cf.ThreadPoolExecutor(max_workers=len(SOURCES) + len(DENSE)) as ex:
        objs = list(ex.map(compile_one, [*DENSE, *SOURCES]))
    tmp = LIB + f".tmp{os.getpid()}"
    r = subprocess.run([cc, *ARCH, "-shared", "-o", tmp, *objs], capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stderr}")
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose=True,
                extra=["-Xptxas", "-v"] if "--ptxas" in sys.argv else []))
