"""Builds the C-ABI CUDA library ``libsqap.so`` in-tree with nvcc for sm_100a."""
from __future__ import annotations

import glob
import os
import re
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libsqap.so")
NVCC = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")

FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "--fmad=true",
         "-Xcompiler", "-fPIC", "-shared"]


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = sources() + glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(os.path.join(HERE, "..", "include", "*.h"))
    return any(os.path.getmtime(d) > t for d in deps)


def register_shortages(log: str, source: str | None = None) -> list[str]:
    """Kernels that move registers between their roles (setmaxnreg) can only be launched with the registers that they were
    written for: kv_prefill_tc_kernel with LAUNCH_REGS a thread. `log` is what ptxas -v said; returns what falls short."""
    if source is None:
        with open(os.path.join(CSRC, "kv_prefill_tc.cu")) as f:
            source = f.read()
    want = int(re.search(r"LAUNCH_REGS = (\d+)", source).group(1))
    used = re.findall(r"Compiling entry function '([^']*kv_prefill_tc_kernel[^']*)'.*?Used (\d+) registers", log, re.S)
    if not used:
        return ["kv_prefill_tc_kernel: not found"]
    return [f"{name}: {n} registers, {want} needed" for name, n in used if int(n) < want]


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not stale():
        return LIB
    extra = os.environ.get("SQAP_NVCC_FLAGS", "").split()
    cmd = [NVCC] + FLAGS + extra + ["-Xptxas", "-v", "-o", LIB + ".tmp"] + sources()
    run = subprocess.run(cmd, stderr=subprocess.PIPE, text=True)
    if verbose or run.returncode:
        sys.stderr.write(run.stderr)
    else:
        sys.stderr.writelines(line + "\n" for line in run.stderr.splitlines() if "warning" in line)
    run.check_returncode()
    short = register_shortages(run.stderr)
    if short:
        raise RuntimeError("the compiler gave a kernel too few registers to be launched: " + "; ".join(short))
    os.replace(LIB + ".tmp", LIB)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
