"""Builds libowl.so (HIP kernels + C ABI) for gfx950 with hipcc, in-tree."""
from __future__ import annotations

import concurrent.futures
import os
import shutil
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
OUT = os.path.join(PKG, "libowl.so")
OBJ = os.path.join(PKG, "_build")
SOURCES = ["owl_splitkv.hip", "owl_splitkv_quant.hip", "owl_splitkv_few.hip", "owl_splitkv_groups.hip", "owl_aux.hip", "owl_steps.hip", "owl_append.hip",
           "owl_groups.hip", "owl_logprobs.hip", "owl_drafter.hip", "owl_probe.hip", "owl_api.hip"]

# -packed-fp32-ops is switched OFF on purpose: packed fp32 VALU forms are not
# to be generated for this target (hipcc's host pass does not know the feature
# and warns; harmless).
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wno-unused-command-line-argument", "-Wno-unknown-attributes", "-Wno-inline-asm",
    "-I" + os.path.join(ROOT, "include"), "-I" + CSRC,
]


def hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found")


def _compile(src: str, extra) -> str:
    obj = os.path.join(OBJ, os.path.splitext(src)[0] + ".o")
    cmd = [hipcc(), *FLAGS, *extra, "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    noise = "is not a recognized feature for this target"
    err = "\n".join(l for l in r.stderr.splitlines() if noise not in l)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed for {src}:\n{err}")
    if err.strip():
        sys.stderr.write(err + "\n")
    return obj


def build_library(extra_flags=(), verbose: bool = False) -> str:
    os.makedirs(OBJ, exist_ok=True)
    with concurrent.futures.ThreadPoolExecutor(max_workers=len(SOURCES)) as ex:
        objs = list(ex.map(lambda s: _compile(s, list(extra_flags)), SOURCES))
    cmd = [hipcc(), "--offload-arch=gfx950", "-shared", "-fPIC", "-o", OUT, *objs]
    subprocess.check_call(cmd)
    if verbose:
        print("built", OUT)
    return OUT


HOST_SOURCES = ["owl_api.hip", "owl_probe.hip"]       # argument checks, planning, hooks: the host logic
HOST_SAN_OUT = os.path.join(PKG, "libowl_hostsan.so")


def build_host_sanitized() -> str:
    """libowl_hostsan.so: the translation units that hold the host logic rebuilt with AddressSanitizer and
    UndefinedBehaviorSanitizer on the HOST side only (device code is not instrumented), linked with the
    ordinary objects of the kernel files.  For host-only tests; needs clang's ASan runtime preloaded."""
    os.makedirs(OBJ, exist_ok=True)
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-sanitize-recover=undefined", "-Xarch_host", "-fno-omit-frame-pointer", "-g"]
    objs = []
    for src in SOURCES:
        obj = os.path.join(OBJ, os.path.splitext(src)[0] + ".o")
        if src in HOST_SOURCES:
            obj = os.path.join(OBJ, os.path.splitext(src)[0] + ".hostsan.o")
            cmd = [hipcc(), *FLAGS, *san, "-c", os.path.join(CSRC, src), "-o", obj]
            r = subprocess.run(cmd, capture_output=True, text=True)
            if r.returncode != 0:
                raise RuntimeError(f"hipcc (host sanitizers) failed for {src}:\n{r.stderr}")
        elif not os.path.exists(obj):
            obj = _compile(src, [])
        objs.append(obj)
    # link only (no device compilation on this line): host sanitizer runtimes, GPU sanitizing explicitly off
    subprocess.check_call([hipcc(), "--offload-arch=gfx950", "-shared", "-fPIC", "-fno-gpu-sanitize",
                           "-fsanitize=address", "-fsanitize=undefined", "-shared-libsan", "-o", HOST_SAN_OUT, *objs])
    return HOST_SAN_OUT


def asan_runtime() -> str:
    """Path of clang's shared AddressSanitizer runtime (to be preloaded into the python process)."""
    out = subprocess.run([hipcc(), "-print-file-name=libclang_rt.asan-x86_64.so"], capture_output=True, text=True)
    path = out.stdout.strip().splitlines()[-1] if out.stdout.strip() else ""
    if not os.path.isabs(path) or not os.path.exists(path):
        import glob
        cands = glob.glob("/opt/rocm/lib/llvm/lib/clang/*/lib/linux/libclang_rt.asan-x86_64.so")
        path = cands[0] if cands else ""
    return path


if __name__ == "__main__":
    build_library(sys.argv[1:], verbose=True)
