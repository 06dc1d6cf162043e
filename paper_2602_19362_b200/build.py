"""Compile the CUDA library in-tree for sm_100a (nvcc cross-compiles without a GPU)."""
from __future__ import annotations

import os
import re
import subprocess
import sys
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "liboapl.so")
SOURCES = ["oapl_api.cu", "step_api.cu", "residual_api.cu", "residual_bwd_bf16.cu", "residual_bwd_f16.cu",
           "residual_bwd_f32.cu"]
DEPS = [*SOURCES, "gemm_sm100.cuh", "small_kernels.cuh", "sm100_ptx.cuh", "sweep_schedule.cuh", "adamw.cuh",
        "logits_ops.cuh", "quantize.cuh", "scaled_matmul.cuh", "residual_host.cuh", "elements.cuh", "host_common.cuh",
        "embedding.cuh", "residual_norm.cuh", "grad_clip.cuh", "logits_adjust.cuh",
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


def _run(commands: list, verbose: bool) -> str:
    """Run the commands side by side; what they reported, one after the other.  Raises if one of them fails."""
    logs = [tempfile.TemporaryFile("w+") for _ in commands]      # not pipes, which would fill up unread
    running = [subprocess.Popen(c, stderr=f) for c, f in zip(commands, logs)]
    codes = [p.wait() for p in running]
    texts = []
    for f, code in zip(logs, codes):
        f.seek(0)
        texts.append(f.read())
        f.close()
        if verbose or code:
            sys.stderr.write(texts[-1])
    for c, code in zip(commands, codes):
        if code:
            raise subprocess.CalledProcessError(code, c)
    return "".join(texts)


def build(force: bool = False, verbose: bool = False) -> str:
    """Build liboapl.so if missing or older than its sources; return its path."""
    if not force and not _stale():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    flags = ["-Xcompiler", "-fPIC", "-std=c++17", "-O3", "-lineinfo", "-Xptxas", "-v",
             "-gencode", "arch=compute_100a,code=sm_100a"]
    # takes the library's place once the check has passed; each process builds one of its own
    with tempfile.TemporaryDirectory(prefix=".build-", dir=HERE) as work:
        new = os.path.join(work, "liboapl.so")
        objects = [os.path.join(work, s + ".o") for s in SOURCES]
        steps = [[nvcc, "-c", *flags, "-o", o, os.path.join(CSRC, s)] for s, o in zip(SOURCES, objects)]
        log = _run(steps, verbose)
        _run([[nvcc, "-shared", *flags, "-o", new, *objects]], verbose)
        check_registers(log, _split_constant())
        os.replace(new, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose=True))
