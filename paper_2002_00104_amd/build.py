"""Builds libpwlq.so (HIP, gfx950) in-tree with hipcc, and the modules that call it from Python with gcc and g++."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libpwlq.so")
CALL_SOURCE = os.path.join(CSRC, "pwlq_call.c")
CALL = os.path.join(HERE, "_pwlq_call" + (sysconfig.get_config_var("EXT_SUFFIX") or ".so"))
BLOCK = os.path.join(CSRC, "block")
BINDING_SOURCE = os.path.join(BLOCK, "binding.cpp")
BINDING = os.path.join(HERE, "_pwlq_block" + (sysconfig.get_config_var("EXT_SUFFIX") or ".so"))
SOURCES = [os.path.join(BLOCK, f) for f in ("library.hip", "adapter.hip", "norm.hip", "pack.hip")]
BLOCK_HEADERS = [os.path.join(BLOCK, f) for f in ("launch.h", "rows.h")] + [
    os.path.join(os.path.dirname(HERE), "include", f) for f in ("pwlq.h", "pwlq_block.h")]
# pwlq_api.hip is part of library.hip
HEADERS = [os.path.join(CSRC, f) for f in sorted(os.listdir(CSRC)) if f.endswith((".h", ".hip"))] + [
           os.path.join(BLOCK, "calls.h"), *BLOCK_HEADERS,
           os.path.join(os.path.dirname(HERE), "include", "pwlq_bench.h")]
OBJECTS = os.path.join(HERE, "_build")

# -ffp-contract=off: the canonical code arithmetic must not be fused; fused
# operations are written explicitly where wanted.  Packed binary32 VALU forms
# are disabled for the device compile.
HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    "-ffp-contract=off", "-fno-fast-math",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
]


# Checking configuration (CPU only): the host side of the library (argument checks,
# tensor table, workspace layout) under AddressSanitizer and
# UndefinedBehaviorSanitizer; the device code is compiled as usual.
LIB_SAN = os.path.join(HERE, "libpwlq_san.so")
HOST_SAN_FLAGS = ["-O1", "-g"] + [f for opt in ("-fsanitize=address", "-fsanitize=undefined",
                                                "-fno-sanitize-recover=all", "-fno-omit-frame-pointer")
                                  for f in ("-Xarch_host", opt)]


def hipcc() -> str:
    for cand in (shutil.which("hipcc"), "/opt/rocm/bin/hipcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found")


def stale(built: str = LIB, sources=None) -> bool:
    if not os.path.exists(built):
        return True
    t = os.path.getmtime(built)
    return any(os.path.getmtime(p) > t for p in sources or SOURCES + HEADERS)


def compile_library(lib: str, flags, force: bool, kind: str = "") -> None:
    """Compiles the sources beside each other, those whose object is older than what it is made of, and links them."""
    os.makedirs(OBJECTS, exist_ok=True)
    running, objects = [], []
    for src in SOURCES:
        obj = os.path.join(OBJECTS, os.path.basename(src) + kind + ".o")
        objects.append(obj)
        headers = HEADERS if src == SOURCES[0] else BLOCK_HEADERS
        if force or stale(obj, [src, *headers]):
            cmd = [hipcc(), *flags, "-c", src, "-o", obj]
            running.append((cmd, subprocess.Popen(cmd)))
    failed = [subprocess.CalledProcessError(p.returncode, cmd) for cmd, p in running if p.wait() != 0]
    if failed:
        raise failed[0]
    subprocess.run([hipcc(), *flags, "-shared", *objects, "-o", lib], check=True)


def build_binding() -> None:
    """The module that calls pwlq_block.h with tensors: torch's headers and libraries, and libpwlq.so beside it."""
    import torch
    from torch.utils import cpp_extension
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-fPIC", "-shared", "-fvisibility=hidden",
                    f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
                    "-I" + sysconfig.get_paths()["include"], *("-isystem" + p for p in cpp_extension.include_paths()),
                    BINDING_SOURCE, "-o", BINDING, "-L" + HERE, "-lpwlq", "-Wl,-rpath,$ORIGIN",
                    *("-L" + p for p in cpp_extension.library_paths()), "-lc10", "-ltorch_cpu", "-ltorch_python"], check=True)


def build(force: bool = True, extra=()) -> str:
    if force or stale():
        compile_library(LIB, [*HIPCC_FLAGS, *extra], force or bool(extra))
    if force or stale(CALL, [CALL_SOURCE]):
        subprocess.run(["gcc", "-O2", "-std=c11", "-Wall", "-Wextra", "-fPIC", "-shared",
                        "-I" + sysconfig.get_paths()["include"], CALL_SOURCE, "-o", CALL], check=True)
    if force or stale(BINDING, [BINDING_SOURCE, *BLOCK_HEADERS]):
        build_binding()
    return LIB


def build_sanitized() -> str:
    flags = [f for f in HIPCC_FLAGS if f != "-O3"]
    compile_library(LIB_SAN, [*flags, *HOST_SAN_FLAGS], True, ".san")
    return LIB_SAN


def sanitizer_runtime() -> str:
    """The shared AddressSanitizer runtime of the compiler hipcc drives ('' if absent)."""
    r = subprocess.run([hipcc(), "-print-file-name=libclang_rt.asan-x86_64.so"],
                       capture_output=True, text=True)
    path = r.stdout.strip()
    if os.path.isabs(path) and os.path.exists(path):
        return path
    import glob
    found = sorted(glob.glob("/opt/rocm/lib/llvm/lib/clang/*/lib/linux/libclang_rt.asan-x86_64.so"))
    return found[-1] if found else ""


if __name__ == "__main__":
    print(build(True, sys.argv[1:]))
