"""Compile the HIP sources under csrc/ for gfx950 into paper_2605_10875_amd/libsol.so.

Each source is compiled to an object file under _build/ (in parallel; an object is reused when it is
newer than its source and every header, unless force=True), then the objects are linked, unless isa.py finds in their
machine code that the compiler has used registers which a kernel takes for itself."""
import glob
import os
import subprocess
from concurrent.futures import ThreadPoolExecutor

if __package__:
    from . import isa
else:                              # run as a script
    import isa

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libsol.so")
TORCH_SRC = os.path.join(CSRC, "sol_torch.cpp")       # the binding's part in C++: an extension module compiled against torch's headers
TORCH_LIB = os.path.join(HERE, "sol_torch.so")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-Wall", "-Wno-unused-function",
         "-Wno-inline-asm"]        # the LDS-direct loads write M0 inside their asm and say so in the clobber list


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.hip")))


def headers():
    return glob.glob(os.path.join(CSRC, "*.h")) + glob.glob(os.path.join(HERE, "..", "include", "*.h"))


def is_stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    return any(os.path.getmtime(p) > t for p in sources() + headers())


def _obj(src):
    return os.path.join(OBJ, os.path.basename(src)[:-4] + ".o")


def _compile(src, verbose):
    cmd = [HIPCC] + FLAGS + ["-c", "-o", _obj(src), src]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)


def build_torch(force: bool = True, verbose: bool = False) -> str:
    if not force and os.path.exists(TORCH_LIB) and os.path.getmtime(TORCH_LIB) >= max(os.path.getmtime(p) for p in [TORCH_SRC] + headers()):
        return TORCH_LIB
    import sysconfig

    import torch
    root = os.path.join(os.path.dirname(torch.__file__))
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}",
           "-isystem", os.path.join(root, "include"), "-isystem", os.path.join(root, "include", "torch", "csrc", "api", "include"),
           "-isystem", sysconfig.get_paths()["include"], "-o", TORCH_LIB, TORCH_SRC, "-L" + os.path.join(root, "lib"), "-ltorch_python",
           "-ltorch_cpu", "-ltorch", "-lc10"]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)
    return TORCH_LIB


def build(force: bool = True, verbose: bool = False) -> str:
    if not force and not is_stale():
        build_torch(False, verbose)
        return LIB
    os.makedirs(OBJ, exist_ok=True)
    newest_header = max(os.path.getmtime(p) for p in headers())
    todo = [s for s in sources()
            if force or not os.path.exists(_obj(s)) or os.path.getmtime(_obj(s)) < max(os.path.getmtime(s), newest_header)]
    jobs = max(1, min(len(todo), int(os.environ.get("MAX_JOBS", os.cpu_count() or 4))))
    with ThreadPoolExecutor(jobs) as ex:
        list(ex.map(lambda s: _compile(s, verbose), todo))
    isa.check_accumulators([_obj(s) for s in sources()])
    cmd = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB] + [_obj(s) for s in sources()]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)
    build_torch(force, verbose)
    return LIB


if __name__ == "__main__":
    import sys
    print(build(force="--force" in sys.argv, verbose=True))
