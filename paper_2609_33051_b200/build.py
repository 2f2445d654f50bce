"""Build libsketchssm.so (the C-ABI CUDA library) in-tree with nvcc for sm_100a."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
import sysconfig

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG_DIR)
CSRC = os.path.join(PKG_DIR, "csrc")
LIB_PATH = os.path.join(PKG_DIR, "libsketchssm.so")
# the operators around the recurrence
LAYER_UNITS = ("api_layer.cu", "conv.cu", "prompt_scan.cu", "prompt_scan_tc.cu", "rms_norm.cu", "scaled_matmul.cu", "scaled_matmul_pair.cu",
               "delta_scan.cu", "delta_scan_tc.cu", "integer_norm.cu", "integer_matmul.cu", "integer_matmul_pair.cu")
# (source, object suffix, extra defines); the decodes are compiled once per (recurrence kind, I/O type)
UNITS = [("api.cu", "", []), ("update.cu", "", []), ("update_cols.cu", "", []), ("update_tc.cu", "", []),
         ("update_tc_ws.cu", "", []), ("update_tc_ws_gdn.cu", "", []), ("update_tc_ws_kda.cu", "", []), ("decode_static.cu", "", []), ("selftest.cu", "", []), ("coef_map.cu", "", []), ("coef_map_pivot.cu", "", []),
         *[(src, f"_k{k}_io{io}", [f"-DSKETCHSSM_GROUP_KIND={k}", f"-DSKETCHSSM_GROUP_IO={io}"])
           for src in ("decode.cu", "decode_split.cu") for k in range(3) for io in range(2)],
         *[(src, "", []) for src in LAYER_UNITS]]
HEADERS = [os.path.join(CSRC, "internal.cuh"), os.path.join(CSRC, "lanegroup.cuh"), os.path.join(CSRC, "tc_common.cuh"),
           os.path.join(CSRC, "state_rows.h"), os.path.join(CSRC, "operand_sets.h"), os.path.join(CSRC, "team_size.h"),
           os.path.join(ROOT, "include", "sketchssm.h")]
LAYER_HEADERS = [os.path.join(CSRC, "layer.cuh"), os.path.join(CSRC, "tma.cuh"), os.path.join(CSRC, "pairs.cuh")]      # of the operators around the recurrence alone


# the extension module that checks tensors and calls the library for the operators around the recurrence
CALLS_SRC = os.path.join(CSRC, "layer_calls.cpp")


def calls_path() -> str:
    """The extension module's file.  It holds for one Python and one torch, which its name says: another one's is never taken for it."""
    import torch
    return os.path.join(PKG_DIR, f"_layer_calls.torch-{torch.__version__}-abi{int(torch.compiled_with_cxx11_abi())}" + sysconfig.get_config_var("EXT_SUFFIX"))


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found; cannot build libsketchssm.so")


def _stale(target: str, deps) -> bool:
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(d) > t for d in deps)


def _calls_command() -> list:
    import torch
    home = os.path.dirname(torch.__file__)
    lib, inc = os.path.join(home, "lib"), os.path.join(home, "include")
    return [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}",
            *[f"-I{d}" for d in (inc, os.path.join(inc, "torch", "csrc", "api", "include"), sysconfig.get_path("include"), os.path.join(ROOT, "include"))],
            CALLS_SRC, "-o", calls_path(), f"-L{lib}", "-ltorch_python", "-ltorch_cpu", "-ltorch", "-lc10", f"-Wl,-rpath,{lib}"]


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile every .cu to an object (parallel-friendly, incremental) and link the shared library."""
    nvcc = _nvcc()
    objdir = os.path.join(PKG_DIR, "build")
    os.makedirs(objdir, exist_ok=True)
    flags = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
             "-Xcompiler", "-fPIC", "-I", os.path.join(ROOT, "include"), "-I", CSRC]
    if verbose:
        flags += ["-Xptxas", "-v"]
    procs, objs = [], []
    if force or _stale(calls_path(), [CALLS_SRC, os.path.join(ROOT, "include", "sketchssm.h")]):
        procs.append(("layer_calls.cpp", subprocess.Popen(_calls_command(), stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    for src, suffix, defs in UNITS:
        sp = os.path.join(CSRC, src)
        obj = os.path.join(objdir, src.replace(".cu", suffix + ".o"))
        objs.append(obj)
        if force or _stale(obj, [sp] + HEADERS + (LAYER_HEADERS if src in LAYER_UNITS else [])):
            procs.append((src + suffix, subprocess.Popen([nvcc, *flags, *defs, "-c", sp, "-o", obj],
                                                stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    failed = []
    for src, pr in procs:
        out, _ = pr.communicate()
        if verbose or pr.returncode != 0:
            sys.stderr.write(out)
        if pr.returncode != 0:
            failed.append(src)
    if any(src != "layer_calls.cpp" for src in failed):
        raise RuntimeError(f"compilation failed: {', '.join(failed)}")
    if force or procs or _stale(LIB_PATH, objs):
        subprocess.check_call([nvcc, "-shared", "-o", LIB_PATH, *objs, "-gencode", "arch=compute_100a,code=sm_100a"])
    if failed:                                          # (the library itself, which decode alone needs, is there)
        raise RuntimeError(f"compilation failed: {', '.join(failed)}")
    return LIB_PATH


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
