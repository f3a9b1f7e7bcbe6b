"""Compile libfwg.so for gfx950 with hipcc (in-tree, next to this file)."""
from __future__ import annotations

import glob
import os
import subprocess
import sys
import sysconfig
import warnings
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libfwg.so")
MARSHAL, MARSHAL_SOURCE = os.path.join(PKG, "_marshal"), os.path.join(CSRC, "fwg_marshal.cpp")  # a module of ops.py
SOURCES = [os.path.join(CSRC, "fwg_host.cpp"), os.path.join(CSRC, "fwg_kernels.hip"),
           os.path.join(CSRC, "fwg_mfma.hip"), os.path.join(CSRC, "fwg_parallel.hip"),
           os.path.join(CSRC, "fwg_parstack.hip"), os.path.join(CSRC, "fwg_parhead.hip"),
           os.path.join(CSRC, "fwg_wave.hip"), os.path.join(CSRC, "fwg_split.hip"),
           os.path.join(CSRC, "fwg_chain.hip"), os.path.join(CSRC, "fwg_wide.hip"),
           os.path.join(CSRC, "fwg_ops.cpp"), os.path.join(CSRC, "fwg_embed.hip"),
           os.path.join(CSRC, "fwg_normq.hip"), os.path.join(CSRC, "fwg_matmulq.hip"),
           os.path.join(CSRC, "fwg_logprob.hip"), os.path.join(CSRC, "fwg_mx.hip"),
           os.path.join(CSRC, "fwg_matmulmx.hip"), os.path.join(CSRC, "fwg_adjust.hip")]
HEADERS = [os.path.join(ROOT, "include", "fwg.h"), os.path.join(CSRC, "fwg_internal.h"),
           os.path.join(CSRC, "fwg_sample.h"), os.path.join(CSRC, "fwg_valu.h"),
           os.path.join(CSRC, "fwg_wave.h"), os.path.join(CSRC, "fwg_par.h"), os.path.join(CSRC, "fwg_mfma_dev.h"),
           os.path.join(CSRC, "fwg_bf16.h"), os.path.join(CSRC, "fwg_chain.h"),
           os.path.join(CSRC, "fwg_xchg.h"), os.path.join(CSRC, "fwg_wide.h"),
           os.path.join(CSRC, "fwg_ops.h"), os.path.join(CSRC, "fwg_ops_dev.h")]

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # packed fp32 instructions stay off: the compiler must not form them from float code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # MFMA accumulators in ordinary VGPRs: avoids AGPR<->VGPR copies around the step loop
    "-mllvm", "-amdgpu-mfma-vgpr-form",
    "-I" + os.path.join(ROOT, "include"), "-I" + CSRC,
]
OBJDIR = os.path.join(PKG, "_build")


def _run(cmd, verbose):
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        sys.stderr.write(r.stdout + r.stderr)
        raise RuntimeError(f"{cmd[0]} failed: " + " ".join(cmd[-3:]))


def marshal_path():
    """Where the module _marshal for this Python and this torch lies (None without torch).  It reads tensors by torch's own
    layouts, so the file's name has both versions and another's module is not found."""
    try:
        import torch
    except ImportError:
        return None
    return f"{MARSHAL}-torch{torch.__version__}{sysconfig.get_config_var('EXT_SUFFIX')}"


def build_marshal(verbose: bool = False) -> None:
    """Compile the module _marshal (host code only); without torch there is nothing to marshal.  ops.py works without the
    module: where it cannot be compiled (no host compiler, no headers) a warning says so.  Modules of other sources or
    versions do not stay."""
    path = marshal_path()
    built = False
    try:
        if path is not None:
            import torch
            from torch.utils.cpp_extension import include_paths, library_paths
            _run([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-shared", "-fPIC",
                  f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}", "-I" + os.path.join(ROOT, "include"),
                  "-I" + sysconfig.get_paths()["include"]] + ["-isystem" + p for p in include_paths()] +
                 ["-o", path + ".tmp", MARSHAL_SOURCE] + ["-L" + p for p in library_paths()] +
                 ["-ltorch_python", "-ltorch_cpu", "-lc10"], verbose)
            os.replace(path + ".tmp", path)
            built = True
    except (ImportError, OSError, RuntimeError) as e:
        warnings.warn(f"the module _marshal was not built: calls of few rows take the host longer ({e})")
    for other in glob.glob(glob.escape(MARSHAL) + "*.so"):
        if not built or other != path:
            os.remove(other)


def build(verbose: bool = False) -> str:
    """Compile every source to an object (in parallel: each is one translation unit with its own
    device code), then link libfwg.so; beside them the module _marshal."""
    os.makedirs(OBJDIR, exist_ok=True)
    objs = [os.path.join(OBJDIR, os.path.basename(src) + ".o") for src in SOURCES]
    jobs = max(1, min(len(SOURCES) + 1, int(os.environ.get("MAX_JOBS", os.cpu_count() or 1))))
    with ThreadPoolExecutor(jobs) as ex:
        for f in [ex.submit(_run, [HIPCC] + FLAGS + ["-c", "-o", o, src], verbose) for src, o in zip(SOURCES, objs)] + \
                [ex.submit(build_marshal, verbose)]:
            f.result()
    tmp = LIB + ".tmp"
    _run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", tmp] + objs, verbose)
    os.replace(tmp, LIB)
    return LIB


def is_stale() -> bool:
    marshal = marshal_path()
    if not os.path.exists(LIB) or (marshal is not None and not os.path.exists(marshal)):
        return True
    t = os.path.getmtime(LIB)
    return any(os.path.getmtime(s) > t for s in SOURCES + HEADERS + [MARSHAL_SOURCE])


if __name__ == "__main__":
    print(build(verbose=True))
