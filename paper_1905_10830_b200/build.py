"""Builds the codec library (CUDA, sm_100a only) in-tree with nvcc.

`python -m paper_1905_10830_b200.build` compiles every source under csrc/ into
`paper_1905_10830_b200/libtc_b200.so` and the layer calls' Python module into `_layers.so`.
Objects are cached under `_build/` by mtime, the module by mtime and by the torch and Python it was
built for.  The codec and the C ABI do not need the module: where it cannot be compiled the library is built all the same.
"""
from __future__ import annotations

import concurrent.futures
import glob
import os
import subprocess
import sys
import sysconfig
import warnings

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
OBJ_DIR = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libtc_b200.so")
LAYERS_SRC, LAYERS = os.path.join(PKG, "binding_layers.cpp"), os.path.join(PKG, "_layers.so")

NVCC = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
COMMON = ["-O3", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo",
          "-Xcompiler", "-fPIC", "-I", os.path.join(ROOT, "include"), "-I", CSRC]


def _sources() -> list[str]:
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")) + glob.glob(os.path.join(CSRC, "*.cpp")))


def _headers_mtime() -> float:
    hdrs = glob.glob(os.path.join(CSRC, "*.h")) + glob.glob(os.path.join(CSRC, "*.cuh")) + \
        glob.glob(os.path.join(ROOT, "include", "*.h"))
    return max(os.path.getmtime(h) for h in hdrs)


def _compile(src: str, verbose: bool) -> str:
    obj = os.path.join(OBJ_DIR, os.path.basename(src) + ".o")
    newest = max(os.path.getmtime(src), _headers_mtime())
    if os.path.exists(obj) and os.path.getmtime(obj) >= newest:
        return obj
    cmd = [NVCC, *COMMON, "-c", src, "-o", obj]
    if verbose:
        cmd.insert(1, "-Xptxas=-v")
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"nvcc failed for {src}:\n{res.stdout}\n{res.stderr}")
    if verbose:
        sys.stderr.write(res.stderr)
    return obj


def layers_built_for() -> tuple[str | None, str]:
    """The torch and Python that the module of the layer calls was built for (None: not known), and those that run."""
    import torch
    here = f"torch {torch.__version__}, {sys.implementation.cache_tag}"
    try:
        with open(LAYERS + ".built") as f:
            return f.read(), here
    except OSError:
        return None, here


def build_layers(force: bool = False) -> str:
    """The module of the layer calls, against this torch's headers; its libraries are loaded by `import torch`."""
    built_for, here = layers_built_for()
    newest = max(os.path.getmtime(LAYERS_SRC), os.path.getmtime(os.path.join(ROOT, "include", "tc.h")))
    if not force and os.path.exists(LAYERS) and os.path.getmtime(LAYERS) >= newest and built_for == here:
        return LAYERS
    import torch
    base = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(NVCC))
    tmp = LAYERS + f".{os.getpid()}.tmp"
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", "-I", os.path.join(ROOT, "include"),
           "-isystem", sysconfig.get_paths()["include"], "-isystem", os.path.join(base, "include"), "-isystem", os.path.join(cuda, "include"),
           LAYERS_SRC, "-o", tmp, "-L", os.path.join(base, "lib"), "-ltorch_python", "-ltorch_cuda", "-ltorch_cpu", "-lc10"]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"g++ failed for {LAYERS_SRC}:\n{res.stdout}\n{res.stderr}")
    os.replace(tmp, LAYERS)
    with open(LAYERS + ".built", "w") as f:
        f.write(here)
    return LAYERS


def build_library(force: bool = False, verbose: bool = False) -> str:
    os.makedirs(OBJ_DIR, exist_ok=True)
    if force:
        for f in glob.glob(os.path.join(OBJ_DIR, "*.o")):
            os.remove(f)
    srcs = _sources()
    with concurrent.futures.ThreadPoolExecutor(max_workers=min(8, len(srcs) + 1)) as pool:
        layers = pool.submit(build_layers, force)
        objs = list(pool.map(lambda s: _compile(s, verbose), srcs))
    if (not os.path.exists(LIB)) or any(os.path.getmtime(o) > os.path.getmtime(LIB) for o in objs):
        tmp = LIB + f".{os.getpid()}.tmp"
        subprocess.check_call([NVCC, "-shared", "-gencode", "arch=compute_100a,code=sm_100a",
                               "-o", tmp, *objs])
        os.replace(tmp, LIB)
    try:
        layers.result()
    except (RuntimeError, OSError, ImportError) as e:
        warnings.warn(f"the layer calls' module was not built, the library was: {e}", RuntimeWarning, stacklevel=2)
    return LIB


def main(args: list[str]) -> int:
    print(build_library(force="--force" in args, verbose="-v" in args))
    try:
        build_layers()
    except (RuntimeError, OSError, ImportError) as e:
        print(e, file=sys.stderr)
        return 1
    return 0


if __name__ == "__main__":
    sys.exit(main(sys.argv[1:]))
