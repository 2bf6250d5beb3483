"""Build libbuddy.so (the HIP library behind include/buddy.h) for gfx950, and
_kv4_bind.so, the argument marshalling of its serving calls (paged 4-bit
cache, norms, 8-bit rows, adapters, sampling).

Each translation unit is compiled by hipcc in parallel, then linked into a
shared library next to this file; the binding is host code of its own,
compiled by g++ against torch's headers and linked to the library.  Run as ``python -m paper_2606_09514_amd.build``.
"""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
SO = os.path.join(HERE, "libbuddy.so")
BIND_SO = os.path.join(HERE, "_kv4_bind.so")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
SOURCES = ["api.hip", "k_route.hip", "k_gemv.hip", "k_attn.hip", "k_mfma.hip", "k_gemm.hip", "prior.hip",
           "kv4.hip", "kv4_attn.hip", "rows8.hip", "linear8.hip", "lora.hip", "sample.hip"]
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Wall",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]


def bind_command(obj: str) -> list:
    """The binding's compile command."""
    import torch
    from torch.utils import cpp_extension
    return [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-Wall",
            f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", "-D__HIP_PLATFORM_AMD__", "-DUSE_ROCM",
            "-I" + sysconfig.get_paths()["include"], *("-isystem" + i for i in cpp_extension.include_paths()),
            "-isystem" + os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "include"),
            "-c", os.path.join(CSRC, "bind.cpp"), "-o", obj]


def bind_link_command(obj: str, out: str) -> list:
    """The binding's link command."""
    import torch
    return [os.environ.get("CXX", "g++"), "-shared", obj, "-o", out, "-L" + HERE, "-l:libbuddy.so",
            "-L" + os.path.join(os.path.dirname(torch.__file__), "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10_hip",
            "-lc10", "-Wl,-rpath,$ORIGIN"]


def start(cmd: list):
    return subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)


def finish(name: str, p, verbose: bool) -> str | None:
    """What a command printed if it failed."""
    out, _ = p.communicate()
    lines = [l for l in out.splitlines() if "packed-fp32-ops" not in l]
    if p.returncode != 0:
        return f"{name}:\n" + "\n".join(lines)
    if verbose and lines:
        print("\n".join(lines))
    return None


def build(verbose: bool = False) -> str:
    """Both libraries.  The binding needs torch's headers and a host compiler;
    libbuddy.so is linked whether or not the binding compiles."""
    objdir = os.path.join(HERE, "_build")
    os.makedirs(objdir, exist_ok=True)
    bind_obj = os.path.join(objdir, "bind.cpp.o")
    try:
        bind, bind_error = start(bind_command(bind_obj)), None
    except (ImportError, OSError) as e:
        bind, bind_error = None, f"bind.cpp:\n{e}"
    procs, objs = [], []
    for src in SOURCES:
        path = os.path.join(CSRC, src)
        if not os.path.exists(path):
            continue
        obj = os.path.join(objdir, src + ".o")
        objs.append(obj)
        procs.append((src, start([HIPCC, *FLAGS, "-c", path, "-o", obj])))
    if bind:
        bind_error = finish("bind.cpp", bind, verbose)
    errors = [e for e in [finish(src, p, verbose) for src, p in procs] if e]
    if errors:
        raise RuntimeError("hipcc failed:\n" + "\n".join(errors + ([bind_error] if bind_error else [])))
    tmp = SO + ".tmp"
    subprocess.run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", *objs, "-o", tmp],
                   check=True)
    os.replace(tmp, SO)
    if not bind_error:
        tmp = BIND_SO + ".tmp"
        bind_error = finish("linking _kv4_bind.so", start(bind_link_command(bind_obj, tmp)), verbose)
    if bind_error:
        # the serving calls raise without it, the others do not need it
        if os.path.exists(BIND_SO):
            os.remove(BIND_SO)
        raise RuntimeError("libbuddy.so is built, its binding is not:\n" + bind_error)
    os.replace(tmp, BIND_SO)
    return SO


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
