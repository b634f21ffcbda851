"""Builds the HIP libraries in-tree for gfx950 with hipcc: libtopk_ragged.so
(the selection), libpaged_kv.so (the paged 8-bit cache around it) and
libserve_step.so (positions, eviction and logits on either side)."""
from __future__ import annotations

import os
import shutil
import subprocess
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
SRC = os.path.join(HERE, "csrc", "topk_ragged.hip")
LIB_PATH = os.path.join(HERE, "libtopk_ragged.so")
PAGED_SRCS = [os.path.join(HERE, "csrc", f"paged_{name}.hip")
              for name in ("tables", "store", "attend", "stream", "prompt", "score")]
PAGED_LIB_PATH = os.path.join(HERE, "libpaged_kv.so")
SERVE_SRCS = [os.path.join(HERE, "csrc", f"serve_{name}.hip") for name in ("rotate", "weigh", "evict", "logits")]
SERVE_LIB_PATH = os.path.join(HERE, "libserve_step.so")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc" if os.path.exists("/opt/rocm/bin/hipcc")
                       else (shutil.which("hipcc") or "hipcc"))

BASE_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # no packed FP32 instructions anywhere in these libraries
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall",
]
FLAGS = [
    *BASE_FLAGS, "-shared",
    # every atomic here is issued by one lane; the wave-level atomic
    # rewrite only adds instructions and waits for returned values at once
    "-mllvm", "-amdgpu-atomic-optimizer-strategy=None",
    # hoisting out of the machine loops only lengthens live ranges in kernels
    # of this size: without it the instance for planned splits takes 96 vector
    # registers instead of 112, the one for item tables 91 instead of 98, the
    # exact kernel 96 instead of 113 (when it was left out: the decode batch
    # 15.82 us instead of 15.87, the captured decode step 105.4 instead of
    # 106.8, 256 rows 24.1 instead of 24.2, chunked prefill 431.6 instead of
    # 430.6)
    "-mllvm", "-disable-machine-licm",
]


def _run(cmd: list[str], verbose: bool) -> subprocess.Popen:
    if verbose:
        print(" ".join(cmd), flush=True)
    return subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)


def _end(proc: subprocess.Popen, verbose: bool) -> None:
    msgs = [ln for ln in proc.communicate()[0].splitlines()
            if ln.strip() and "packed-fp32-ops" not in ln]
    if proc.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + "\n".join(msgs))
    if verbose and msgs:
        print("\n".join(msgs))


def _build_of(srcs: list[str], path: str, verbose: bool) -> str:
    """A library of several sources, each compiled by itself."""
    with tempfile.TemporaryDirectory() as tmp:
        objs = [os.path.join(tmp, os.path.basename(s) + ".o") for s in srcs]
        procs = [_run([HIPCC, *BASE_FLAGS, "-c", s, "-o", o], verbose) for s, o in zip(srcs, objs)]
        try:
            for p in procs:
                _end(p, verbose)
        finally:
            for p in procs:
                if p.poll() is None:
                    p.kill()
        _end(_run([HIPCC, "--offload-arch=gfx950", "-shared", "-o", path + ".tmp", *objs], verbose), verbose)
    os.replace(path + ".tmp", path)
    return path


def build_paged(verbose: bool = False) -> str:
    return _build_of(PAGED_SRCS, PAGED_LIB_PATH, verbose)


def build_serve(verbose: bool = False) -> str:
    return _build_of(SERVE_SRCS, SERVE_LIB_PATH, verbose)


def build(verbose: bool = False) -> str:
    topk = _run([HIPCC, *FLAGS, "-o", LIB_PATH + ".tmp", SRC], verbose)
    try:
        build_paged(verbose)
        build_serve(verbose)
    finally:
        _end(topk, verbose)
    os.replace(LIB_PATH + ".tmp", LIB_PATH)
    return LIB_PATH


if __name__ == "__main__":
    print(build(verbose=True))
