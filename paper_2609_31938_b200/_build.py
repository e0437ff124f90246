"""In-tree build of the CUDA library (nvcc, sm_100a only): one object per source, built side by side, one library."""
from __future__ import annotations

import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.environ.get("CCV3D_LIB") or os.path.join(HERE, "libccv3d.so")   # (CCV3D_LIB: another build of the library, for diagnosis)
HEADER = os.path.join("..", "..", "include", "ccv3d.h")
SOURCES = {   # source -> the files its object depends on
    "ccv3d_api.cu": ["ccv3d_simt.cuh", "ccv3d_tc.cuh", "ccv3d_tc_layout.cuh", "ccv3d_tc_ptx.cuh", "ccv3d_tc_conv.cuh",
                     "ccv3d_tc_pointwise.cuh", "ccv3d_host_common.cuh", "ccv3d_host_tc.cuh", "ccv3d_host_ring.cuh", HEADER],
    "ccv3d_tokens.cu": ["ccv3d_tokens_common.cuh", "ccv3d_tokens_norm.cuh", "ccv3d_tokens_append.cuh",
                        "ccv3d_tokens_softmax.cuh", "ccv3d_tokens_attend.cuh", "ccv3d_tokens_attend_step.cuh",
                        "ccv3d_tokens_attend_tile.cuh", "ccv3d_tokens_host.cuh", "ccv3d_tc_ptx.cuh", HEADER],
    "ccv3d_group_norm.cu": ["ccv3d_tokens_common.cuh", "ccv3d_tokens_activation.cuh", "ccv3d_tokens_group_norm.cuh",
                            "ccv3d_tokens_host.cuh", HEADER],
    "ccv3d_linear.cu": ["ccv3d_tokens_common.cuh", "ccv3d_tokens_activation.cuh", "ccv3d_tokens_linear.cuh", "ccv3d_tokens_host.cuh",
                        "ccv3d_tc_ptx.cuh", HEADER],
    "ccv3d_decay.cu": ["ccv3d_tokens_common.cuh", "ccv3d_tokens_decay.cuh", "ccv3d_tokens_decay_tile.cuh", "ccv3d_tokens_host.cuh",
                       "ccv3d_tc_ptx.cuh", HEADER],
}

NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "-Xcompiler", "-fPIC"]


def _obj(src: str) -> str:
    return LIB + "." + os.path.splitext(src)[0] + ".o"


def _stale(target: str, files) -> bool:
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(f) > t for f in files)


def stale() -> bool:
    return any(_stale(LIB, [os.path.join(CSRC, f) for f in [s, *deps]]) for s, deps in SOURCES.items())


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile libccv3d.so next to this file; returns its path.  Without `force` only what changed is compiled."""
    if force or stale():
        nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
        running = []
        for src, deps in SOURCES.items():
            if force or _stale(_obj(src), [os.path.join(CSRC, f) for f in [src, *deps]]):
                cmd = [nvcc] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + \
                      ["-c", "-o", _obj(src), os.path.join(CSRC, src)]
                running.append((cmd, subprocess.Popen(cmd)))
        for cmd, p in running:
            if p.wait() != 0:
                for _, other in running:
                    other.wait()
                raise subprocess.CalledProcessError(p.returncode, cmd)
        subprocess.run([nvcc] + NVCC_FLAGS + ["-shared", "-o", LIB + ".tmp"] + [_obj(s) for s in SOURCES], check=True)
        os.replace(LIB + ".tmp", LIB)
    return LIB


if __name__ == "__main__":
    import sys
    print(build(force="--changed" not in sys.argv, verbose=True))
