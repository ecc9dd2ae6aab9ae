"""Build the route-scoring library (libhwr) in-tree with nvcc for sm_103a.

Each .cu file of csrc/ is compiled to an object in parallel, then linked into
one shared library with the CUDA runtime linked statically, so that loading
it needs no libcudart on the library path.  The output goes to
``_build/libhwr_<machine>.so`` next to this file (git-ignored).  The torch
binding of the operators (csrc/ops_torch.cpp, g++) is compiled beside it into
``_build/hwr_torch_<machine>.so``, which links the library; the library needs
nvcc alone, and is built where torch is not installed too.
"""
from __future__ import annotations

import importlib.util
import os
import platform
import shutil
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
OUT_DIR = os.path.join(HERE, "_build")
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]

# Per-file flags: the SIMT kernels follow the canonical fp32 order, so no
# multiply-add contraction may be introduced there.
SOURCES = {
    "hwr_api.cu": [],
    "k_simt.cu": ["--fmad=false"],
    "k_tc.cu": [],
    "hwr_noalloc.cu": [],
    "ops_api.cu": [],
    "k_group.cu": [],
    "k_ops.cu": [],
    "k_few.cu": [],
}


def lib_path() -> str:
    return os.path.join(OUT_DIR, f"libhwr_{platform.machine()}.so")


def torch_path() -> str:
    return os.path.join(OUT_DIR, f"hwr_torch_{platform.machine()}.so")


def _torch_dir():
    """Where torch is installed; None where it is not."""
    spec = importlib.util.find_spec("torch")
    if spec is None or not spec.submodule_search_locations:
        return None
    return list(spec.submodule_search_locations)[0]


def _torch_commands(torch: str, out: str):
    """Compile and link commands of the torch binding."""
    obj = os.path.join(OUT_DIR, f"ops_torch_{platform.machine()}.o")
    compile_ = ["g++", "-O2", "-std=c++17", "-fPIC", "-fvisibility=hidden", "-I", INCLUDE,
                "-isystem", os.path.join(torch, "include"),
                "-isystem", os.path.join(torch, "include", "torch", "csrc", "api", "include"),
                "-isystem", sysconfig.get_paths()["include"],
                "-c", os.path.join(CSRC, "ops_torch.cpp"), "-o", obj]
    lib = os.path.join(torch, "lib")
    # (the library by its name, found beside the binding: the folder may move)
    link = ["g++", "-shared", obj, "-o", out, "-L", OUT_DIR, "-l:" + os.path.basename(lib_path()),
            "-L", lib, "-ltorch_python", "-ltorch_cpu", "-lc10", "-Wl,-rpath,$ORIGIN"]
    return compile_, link


def _nvcc() -> str:
    p = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(p):
        raise RuntimeError("nvcc not found")
    return p


def _stale(out: str) -> bool:
    outs = [out] + ([torch_path()] if _torch_dir() else [])
    if not all(os.path.exists(o) for o in outs):
        return True
    t = min(os.path.getmtime(o) for o in outs)
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)]
    deps += [os.path.join(INCLUDE, f) for f in os.listdir(INCLUDE)]
    deps.append(os.path.abspath(__file__))
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False, ptxas_info: bool = False) -> str:
    """Compile and link libhwr, and the torch binding where torch is installed;
    returns the path of libhwr.  A binding that does not build leaves libhwr in
    place (and raises)."""
    out = lib_path()
    if not force and not _stale(out):
        return out
    os.makedirs(OUT_DIR, exist_ok=True)
    nvcc = _nvcc()
    common = ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC",
              "-I", INCLUDE, "-I", CSRC, *ARCH]
    if ptxas_info:
        common += ["-Xptxas", "-v"]
    procs, objs = [], []

    def compile_(src, cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE,
                                            stderr=subprocess.STDOUT, text=True)))

    for src, extra in SOURCES.items():
        obj = os.path.join(OUT_DIR, src.replace(".cu", f"_{platform.machine()}.o"))
        objs.append(obj)
        compile_(src, [nvcc, *common, *extra, "-c", os.path.join(CSRC, src), "-o", obj])
    torch = _torch_dir()
    if torch:
        torch_out = torch_path() + ".tmp"
        torch_compile, torch_link = _torch_commands(torch, torch_out)
        compile_("ops_torch.cpp", torch_compile)
    errors = {}
    for src, p in procs:
        text, _ = p.communicate()
        if p.returncode != 0:
            errors[src] = f"--- {src}\n{text}"
        elif verbose or ptxas_info:
            sys.stdout.write(text)
    if any(src in errors for src in SOURCES):
        raise RuntimeError("nvcc failed:\n" + "\n".join(errors.values()))
    tmp = out + ".tmp"
    link = [nvcc, "-shared", *ARCH, "-cudart", "static", *objs, "-o", tmp]
    subprocess.run(link, check=True)
    os.replace(tmp, out)
    if errors:
        raise RuntimeError("the operators' torch binding does not compile:\n" + "\n".join(errors.values()))
    if torch:
        subprocess.run(torch_link, check=True)
        os.replace(torch_out, torch_path())
    return out


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv,
                ptxas_info="--ptxas" in sys.argv))
