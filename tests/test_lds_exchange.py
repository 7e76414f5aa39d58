"""Lanes of a wave that pass data on through LDS without a workgroup's barrier: the hardware keeps the order of one wave's accesses, and the compiler has to be told by
fences, without which it may move a thread's read ahead of its own store to another address.  Read from the device code before and behind the optimizer.  CPU only."""
import os
import re
import subprocess

import pytest

from paper_2512_18453_amd import build


def functions(source, tmp_path, flags=()):
    """{function: what its instructions do to LDS, in the order of the text}: S store, L load, R and A release and acquire fences, W a wave's barrier, B a workgroup's."""
    out = str(tmp_path / "code.ll")
    subprocess.run(["hipcc"] + build.COMMON + build.DEVICE + build.PRELOAD + [*flags, "-S", "-emit-llvm", "--offload-device-only", os.path.join(build.SRC, source), "-o", out],
                   check=True, capture_output=True)
    with open(out) as f:
        text = f.read()
    found = {}
    for m in re.finditer(r"^define [^\n]*@(\w+)\(.*?^}", text, re.M | re.S):
        ops = ""
        for ln in m[0].splitlines():
            if "addrspace(3)" in ln and re.search(r"= load ", ln):
                ops += "L"
            elif "addrspace(3)" in ln and re.match(r"\s*store ", ln):
                ops += "S"
            elif re.match(r"\s*fence ", ln):
                ops += "R" if " release" in ln else "A" if " acquire" in ln else "RA"
            elif "call" in ln and "llvm.amdgcn.wave.barrier" in ln:
                ops += "W"
            elif "call" in ln and "llvm.amdgcn.s.barrier" in ln:
                ops += "B"
        found[m[1]] = ops
    return found


@pytest.mark.parametrize("source", ["q4_linear.hip", "logprobs.hip"])
def test_barriers_of_a_wave_have_their_fences(source, tmp_path):
    barriers = 0
    for name, ops in functions(source, tmp_path, ("-Xclang", "-disable-llvm-passes")).items():
        barriers += ops.count("W")
        assert ops.count("W") == ops.count("RWA"), (name, ops)
    assert barriers > 0


def test_rows_operand_of_few_rows(tmp_path):
    # here all that is read from LDS was written by other lanes
    kernels = {name: ops for name, ops in functions("q4_linear.hip", tmp_path).items() if "few_rows" in name}
    assert kernels
    for name, ops in kernels.items():
        assert "L" in ops and not re.search("SL|LS", ops), (name, ops)
