"""Builds libfira.so (the C-ABI library) in-tree with nvcc for sm_100a, and the binding's reading of tensor lists."""
from __future__ import annotations

import glob
import hashlib
import os
import subprocess
import sys
import sysconfig

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(PKG_DIR, "csrc")
LIB_PATH = os.path.join(PKG_DIR, "libfira.so")
SOURCES = ["fira_api.cu", "step_simt.cu", "step_tc.cu", "refresh.cu", "part_gemm.cu", "part_back.cu", "part_project.cu", "noalloc.cu", "adam_dense.cu",
           "grad_clip.cu", "embedding.cu", "layer_norm.cu"]
NVCC_FLAGS = ["-O3", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo",
              "-Xcompiler", "-fPIC", "-Xcompiler", "-fvisibility=hidden", "--expt-relaxed-constexpr"]


# The binding's reading of tensor lists (grad_list.cpp), named for the interpreter that it is built for.
LISTS_PATH = os.path.join(PKG_DIR, "_native_lists" + sysconfig.get_config_var("EXT_SUFFIX"))
LISTS_KEY_PATH = os.path.join(PKG_DIR, "_build", "native_lists.key")
HEADER = os.path.join(os.path.dirname(PKG_DIR), "include", "fira.h")


def _lists_key(torch) -> str:
    """What the module is made from: its source, the header whose descriptors it writes, torch and the interpreter."""
    key = hashlib.sha256()
    for path in (os.path.join(CSRC, "grad_list.cpp"), HEADER):
        with open(path, "rb") as f:
            key.update(f.read() + b"\0")
    key.update(f"{torch.__version__} {int(torch._C._GLIBCXX_USE_CXX11_ABI)} {os.path.basename(LISTS_PATH)}".encode())
    return key.hexdigest()


def _build_lists(force: bool) -> None:
    """Compiles the binding's reading of tensor lists against torch's headers, anew where anything that it is made from has
    changed.  It is a matter of speed alone: where it cannot be built, that is said, nothing older is left in its place, and
    the binding reads lists in Python."""
    import torch
    key = _lists_key(torch)
    if not force and os.path.exists(LISTS_PATH) and os.path.exists(LISTS_KEY_PATH):
        with open(LISTS_KEY_PATH) as f:
            if f.read() == key:
                return
    for old in glob.glob(os.path.join(os.path.dirname(LISTS_PATH), "_native_lists*.so")) + [LISTS_KEY_PATH]:
        if os.path.exists(old):
            os.remove(old)
    root, made = os.path.dirname(torch.__file__), f"{LISTS_PATH}.{os.getpid()}"
    cmd = ["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-fvisibility=hidden",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", f'-DFIRA_LISTS_TORCH="{torch.__version__}"',
           f"-I{root}/include", f"-I{root}/include/torch/csrc/api/include", f"-I{sysconfig.get_paths()['include']}",
           os.path.join(CSRC, "grad_list.cpp"), "-o", made,
           f"-L{root}/lib", "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10", f"-Wl,-rpath,{root}/lib"]
    try:
        done = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
        said = done.stdout if done.returncode else None
    except OSError as e:
        said = str(e)
    if said is not None:
        if os.path.exists(made):
            os.remove(made)
        sys.stderr.write(f"--- not built: {LISTS_PATH} (lists of tensors are read in Python)\n{said}\n")
        return
    os.replace(made, LISTS_PATH)
    os.makedirs(os.path.dirname(LISTS_KEY_PATH), exist_ok=True)
    with open(LISTS_KEY_PATH, "w") as f:
        f.write(key)


def _nvcc() -> str:
    cand = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "bin", "nvcc")
    return cand if os.path.exists(cand) else "nvcc"


def needs_build() -> bool:
    if not os.path.exists(LIB_PATH):
        return True
    t = os.path.getmtime(LIB_PATH)
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if not f.endswith(".cpp")]
    deps.append(HEADER)
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    """Compiles every .cu of the library to objects (in parallel) and links the
    shared library next to this file.  Returns the library path."""
    _build_lists(force)
    if not force and not needs_build():
        return LIB_PATH
    obj_dir = os.path.join(PKG_DIR, "_build")
    os.makedirs(obj_dir, exist_ok=True)
    procs = []
    objs = []
    extra = ["-Xptxas", "-v"] if verbose else []
    for src in SOURCES:
        obj = os.path.join(obj_dir, src.replace(".cu", ".o"))
        objs.append(obj)
        cmd = [_nvcc(), *NVCC_FLAGS, *extra, "-c", os.path.join(CSRC, src), "-o", obj]
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT,
                                            text=True)))
    failed = False
    for src, p in procs:
        out, _ = p.communicate()
        if p.returncode != 0 or verbose:
            sys.stderr.write(f"--- nvcc {src}\n{out}\n")
        failed = failed or p.returncode != 0
    if failed:
        raise RuntimeError("nvcc failed")
    link = [_nvcc(), "-shared", "-o", LIB_PATH, *objs, "-lcudart", "-lcuda"]
    subprocess.run(link, check=True)
    return LIB_PATH


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
