"""Builds libstc.so in-tree with nvcc for sm_100a (no JIT cache, no torch extension)."""
from __future__ import annotations

import os
import subprocess
import sys
from pathlib import Path

PKG = Path(__file__).resolve().parent
ROOT = PKG.parent
CSRC = PKG / "csrc"
LIB = PKG / "libstc.so"
SOURCES = ["stc_api.cu", "page_meta.cu", "quest_select.cu", "quest_select_static.cu", "page_class.cu", "route_pack.cu", "append.cu", "rope.cu", "route_pages.cu", "router.cu", "query_bias.cu", "decode_attn.cu", "scored_attn.cu", "prefix_attn.cu"]
NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-std=c++17", "-lineinfo",
    "-Xcompiler", "-fPIC",
    "-I", str(ROOT / "include"), "-I", str(CSRC),
]


ARGS_SRC = CSRC / "tensor_args.cpp"


def _build_args(force: bool = False) -> None:
    """The binding's argument check (a CPython module against the headers of the installed torch), in-tree.  It is optional: where it
    does not compile the binding checks in Python."""
    if str(ROOT) not in sys.path:                # run by its path
        sys.path.insert(0, str(ROOT))
    from paper_2604_21335_b200 import binding
    lib = binding.args_library()
    if not force and lib.exists() and lib.stat().st_mtime >= ARGS_SRC.stat().st_mtime:
        return
    import sysconfig

    import torch
    root = Path(torch.__file__).resolve().parent
    include = [root / "include", root / "include" / "torch" / "csrc" / "api" / "include", sysconfig.get_paths()["include"]]
    tmp = lib.with_name(f"{lib.name}.{os.getpid()}.tmp")
    try:
        subprocess.check_call([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared",
                               f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
                               *[f"-I{p}" for p in include], str(ARGS_SRC), "-o", str(tmp), f"-L{root / 'lib'}",
                               "-ltorch_python", "-ltorch_cpu", "-lc10"])
    except (OSError, subprocess.CalledProcessError) as e:
        sys.stderr.write(f"the native argument check was not built, the binding checks in Python: {e}\n")
        tmp.unlink(missing_ok=True)
        lib.unlink(missing_ok=True)              # of an older source
        return
    os.replace(tmp, lib)


def _stale() -> bool:
    if not LIB.exists():
        return True
    t = LIB.stat().st_mtime
    deps = list(CSRC.glob("*.cu")) + list(CSRC.glob("*.cuh")) + list((ROOT / "include").glob("*.h"))
    return any(p.stat().st_mtime > t for p in deps)


def build(force: bool = False, verbose: bool = False) -> Path:
    """Compile every CUDA source into one shared library; returns its path."""
    _build_args(force)
    if not force and not _stale():
        return LIB
    nvcc = os.environ.get("NVCC", "nvcc")
    objs = []
    procs = []
    bdir = PKG / "_build"
    bdir.mkdir(exist_ok=True)
    for src in SOURCES:
        obj = bdir / (src + ".o")
        cmd = [nvcc, *NVCC_FLAGS, "-c", str(CSRC / src), "-o", str(obj)]
        if verbose:
            cmd.insert(1, "-Xptxas=-v")
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
        objs.append(str(obj))
    failed = False
    for src, p in procs:
        out, _ = p.communicate()
        if out.strip() and (verbose or p.returncode != 0):
            sys.stderr.write(f"--- {src}\n{out}\n")
        failed |= p.returncode != 0
    if failed:
        raise RuntimeError("nvcc failed")
    tmp = LIB.with_suffix(f".{os.getpid()}.tmp")
    subprocess.check_call([nvcc, "-shared", "-o", str(tmp), *objs, "-lcudart", "-ldl"])
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    build(force=True, verbose="-v" in sys.argv)
    print(LIB)
