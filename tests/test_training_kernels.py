"""Registers and scratch of the kernels of 8-bit float layers and of dropout, and the fences around what the lanes of a wave pass on through LDS, from the compiled code.
CPU only."""
import os
import re
import subprocess

import pytest

from paper_2512_18453_amd import build
from tests.test_kernel_resources import TOOLS
from tests.test_lds_exchange import functions


def resources(source, tmp_path):
    """{kernel's symbol: (vector registers, bytes of scratch)}"""
    obj = os.path.join(build.OBJ, source + ".o")
    if not os.path.exists(obj):
        pytest.skip("objects are not built here")
    bundle, code = str(tmp_path / "bundle"), str(tmp_path / "code")
    subprocess.check_call(["objcopy", "-O", "binary", "--only-section=.hip_fatbin", "--set-section-flags", ".hip_fatbin=alloc", obj, bundle])
    subprocess.check_call([f"{TOOLS}/clang-offload-bundler", "--unbundle", "--type=o", "--targets=hipv4-amdgcn-amd-amdhsa--gfx950",
                           f"--input={bundle}", f"--output={code}"])
    notes = subprocess.check_output([f"{TOOLS}/llvm-readelf", "--notes", code], text=True)

    def every(field, value):
        return re.findall(rf"^    \.{field}: +({value})$", notes, re.M)
    return dict(zip(every("name", r"\S+"), zip(map(int, every("vgpr_count", r"\d+")), map(int, every("private_segment_fixed_size", r"\d+")), strict=True), strict=True))


@pytest.mark.parametrize("source,most", [("f8_matmul.hip", 256), ("f8_layout.hip", 256), ("dropout.hip", 64)])
def test_resources(source, most, tmp_path):
    got = resources(source, tmp_path)
    assert got
    for name, (registers, scratch) in got.items():
        assert registers <= most and scratch == 0, (name, registers, scratch)


@pytest.mark.parametrize("source", ["f8_matmul.hip", "f8_layout.hip"])
def test_barriers_of_a_wave_have_their_fences(source, tmp_path):
    barriers = 0
    for name, ops in functions(source, tmp_path, ("-Xclang", "-disable-llvm-passes")).items():
        barriers += ops.count("W")
        assert ops.count("W") == ops.count("RWA"), (name, ops)
    assert barriers > 0
