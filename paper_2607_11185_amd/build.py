"""Build libseg.so (HIP, gfx950) in-tree with hipcc."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(HERE, "libseg.so")
SOURCES = ["seg_layout.hip", "seg_attn.hip", "seg_logprob.hip", "seg_layer.hip",
           "seg_mrope.hip", "seg_act.hip", "seg_glu.hip", "seg_fp8.hip", "seg_fp8_gemm.hip", "seg_top.hip",
           "seg_distill.hip", "seg_profile.hip"]

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # no packed-fp32 instructions in device code
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function", "-Wno-unused-variable",
]


# Host-code sanitizers (AddressSanitizer + UndefinedBehaviorSanitizer) for a
# CPU-side check build: every flag applies to the host compilation only, the
# device code is built as usual.
SANITIZE_FLAGS = [
    "-Xarch_host", "-fsanitize=address",
    "-Xarch_host", "-fsanitize=undefined",
    "-Xarch_host", "-fno-sanitize-recover=undefined",
    "-Xarch_host", "-fno-omit-frame-pointer", "-g",
]
SANITIZE_LINK = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
                 "-Xarch_host", "-shared-libasan"]
SANITIZED_LIB = os.path.join(HERE, "_build", "sanitize", "libseg.so")


def build(verbose: bool = False, jobs: int = 3, sanitize: bool = False) -> str:
    """Compile every HIP source and link libseg.so next to this file; with
    `sanitize`, the host-sanitizer build at SANITIZED_LIB instead (load it
    with the ASan runtime preloaded, e.g. through SEG_LIB_PATH)."""
    objdir = os.path.join(HERE, "_build", "sanitize") if sanitize else os.path.join(HERE, "_build")
    out = SANITIZED_LIB if sanitize else LIB
    flags = FLAGS + SANITIZE_FLAGS if sanitize else FLAGS
    if sanitize:
        flags = [f if f != "-O3" else "-O1" for f in flags]
    os.makedirs(objdir, exist_ok=True)
    procs = []
    objs = []
    for src in SOURCES:
        obj = os.path.join(objdir, src.replace(".hip", ".o"))
        objs.append(obj)
        cmd = [HIPCC, *flags, "-I", INCLUDE, "-I", CSRC, "-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT)))
        if len(procs) >= jobs:
            _wait(procs.pop(0))
    for p in procs:
        _wait(p)
    tmp = out + ".tmp"
    cmd = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", *(SANITIZE_LINK if sanitize else []),
           "-o", tmp, *objs]
    subprocess.run(cmd, check=True)
    os.replace(tmp, out)
    return out


def asan_runtime() -> str:
    """Path of the compiler's shared AddressSanitizer runtime."""
    clang = os.path.join(os.path.dirname(os.path.realpath(HIPCC)), "..", "llvm", "bin", "clang")
    if not os.path.exists(clang):
        clang = "/opt/rocm/llvm/bin/clang"
    return subprocess.run([clang, "-print-file-name=libclang_rt.asan-x86_64.so"], check=True,
                          capture_output=True, text=True).stdout.strip()


def _wait(item):
    src, p = item
    out, _ = p.communicate()
    text = out.decode(errors="replace")
    lines = [l for l in text.splitlines() if "packed-fp32-ops" not in l]
    if p.returncode != 0:
        sys.stderr.write("\n".join(lines) + "\n")
        raise RuntimeError(f"hipcc failed on {src}")
    if lines:
        sys.stderr.write("\n".join(lines) + "\n")


if __name__ == "__main__":
    print(build(verbose=True, sanitize="--sanitize" in sys.argv))
