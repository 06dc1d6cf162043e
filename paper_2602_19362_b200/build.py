"""Compile the CUDA library in-tree for sm_100a (nvcc cross-compiles without a GPU)."""
from __future__ import annotations

import os
import re
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "liboapl.so")
SOURCES = ["oapl_api.cu"]
DEPS = ["oapl_api.cu", "gemm_sm100.cuh", "small_kernels.cuh", "sm100_ptx.cuh", "sweep_schedule.cuh", "adamw.cuh",
        "logits_ops.cuh", "quantize.cuh", "scaled_matmul.cuh",
        os.path.join("..", "..", "include", "oapl.h")]


# The kernel that divides its launch's registers among its warps, and where the number that it counts on stands.
SPLIT_KERNEL, SPLIT_SOURCE, SPLIT_CONSTANT = "scaled_matmul_kernel", "scaled_matmul.cuh", "kSmRegs"


def check_registers(log: str, want: int) -> None:
    """Raise unless every instance of SPLIT_KERNEL in ptxas's report has `want` registers: with fewer, the split would
    wait for registers that the launch does not have, so the library refuses to launch it."""
    got = re.findall(r"Compiling entry function '(\S*%s\S*)'.*?Used (\d+) registers" % SPLIT_KERNEL, log, re.S)
    wrong = {name: int(n) for name, n in got if int(n) != want}
    if not got or wrong:
        raise RuntimeError(f"{SPLIT_SOURCE}: this compiler gives {SPLIT_KERNEL} {wrong or 'no reported'} registers, "
                           f"its register split counts on {SPLIT_CONSTANT} = {want}")


def _split_constant() -> int:
    with open(os.path.join(CSRC, SPLIT_SOURCE)) as f:
        return int(re.search(r"\b%s = (\d+)" % SPLIT_CONSTANT, f.read()).group(1))


def _stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    return any(os.path.getmtime(os.path.join(CSRC, f)) > t for f in DEPS)


def build(force: bool = False, verbose: bool = False) -> str:
    """Build liboapl.so if missing or older than its sources; return its path."""
    if not force and not _stale():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    # takes the library's place once the check has passed; each process builds one of its own
    new = os.path.join(HERE, f".liboapl-{os.getpid()}.so")
    cmd = [nvcc, "-shared", "-Xcompiler", "-fPIC", "-std=c++17", "-O3", "-lineinfo", "-Xptxas", "-v",
           "-gencode", "arch=compute_100a,code=sm_100a", "-o", new]
    cmd += [os.path.join(CSRC, s) for s in SOURCES]
    try:
        done = subprocess.run(cmd, stderr=subprocess.PIPE, text=True)
        if verbose or done.returncode:
            sys.stderr.write(done.stderr)
        done.check_returncode()
        check_registers(done.stderr, _split_constant())
        os.replace(new, LIB)
    finally:
        if os.path.exists(new):
            os.remove(new)
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose=True))
