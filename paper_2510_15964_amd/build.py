"""Build in-tree: the HIP library liblx_sparse.so (gfx950) and the native part of its Python binding, _lx_call.<ABI tag>.so."""
from __future__ import annotations

import importlib.machinery
import os
import subprocess
import sys
import sysconfig
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "liblx_sparse.so")
# The tag of this interpreter is part of the name: another one, whose objects are laid out otherwise, finds no file.
CALL = os.path.join(HERE, "_lx_call" + importlib.machinery.EXTENSION_SUFFIXES[0])
SOURCES = ["lx_api.hip", "compact.hip", "ffn_f32.hip", "ffn_bf16.hip", "predict_bf16.hip", "lora_bf16.hip",
           "attn_bf16.hip", "attn_f32.hip", "probe.hip", "lx_step_api.hip", "rope.hip", "clip.hip", "score_bf16.hip",
           "score_token.hip", "score_plain.hip"]
# -Wno-inline-asm: the DMA helpers name m0 (a register the compiler reserves) as clobbered, which
# is the point, and clang warns about every such statement
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Wall", "-Wno-inline-asm",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]


def _run(cmd, out) -> None:
    r = subprocess.run(cmd, capture_output=True, text=True)
    err = "\n".join(l for l in r.stderr.splitlines()
                    if "not a recognized feature" not in l)
    if r.returncode != 0:
        if os.path.exists(out):
            os.remove(out)          # never leave a stale library behind a failed build
        raise RuntimeError(f"{os.path.basename(cmd[0])} failed:\n" + err)
    if err.strip():
        sys.stderr.write(err + "\n")


def build(verbose: bool = False) -> str:
    _run(["g++", "-O2", "-std=c++17", "-Wall", "-shared", "-fPIC", "-fvisibility=hidden",
          "-I" + sysconfig.get_paths()["include"], os.path.join(CSRC, "lx_call.cpp"), "-o", CALL], CALL)
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    extra = ["-Rpass-analysis=kernel-resource-usage"] if verbose else []
    # source by source, some at a time (all in one command take five minutes), the longest first
    with tempfile.TemporaryDirectory() as tmp, ThreadPoolExecutor(min(8, os.cpu_count() or 1)) as pool:
        made = {s: os.path.join(tmp, s + ".o") for s in SOURCES}
        by_size = sorted(SOURCES, key=lambda s: os.path.getsize(os.path.join(CSRC, s)), reverse=True)
        for _ in pool.map(lambda s: _run([hipcc, *FLAGS, *extra, "-c", os.path.join(CSRC, s), "-o", made[s]], LIB), by_size):
            pass
        _run([hipcc, "--offload-arch=gfx950", "-shared", "-Wl,--no-undefined", *made.values(), "-o", LIB], LIB)
    return LIB


def ensure() -> None:
    """Builds if any of what the package loads is not there."""
    if not (os.path.exists(LIB) and os.path.exists(CALL)):
        build()


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
