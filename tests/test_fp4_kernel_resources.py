"""Registers of the products' kernels with packed FP4 weights, checked at compile time (no GPU): the largest blocks hold 128 sums, a step's weights and
activations in nearly all registers that two wavefronts a SIMD leave, and their halves take turns only while both are resident."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2511_10909_amd", "csrc")


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")
@pytest.mark.parametrize("source,kernel,count", [("matmul_fp4_tiled", "tiled_kernel", 44), ("matmul_fp4", "stream_kernel", 74)])
def test_products_need_no_scratch_memory(source, kernel, count):
    cmd = ["hipcc", "-c", os.path.join(CSRC, source + ".hip"), "-o", os.devnull, "--offload-arch=gfx950", "--cuda-device-only", "-O3", "-fPIC",
           "-std=c++17", "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
           "-Rpass-analysis=kernel-resource-usage"]
    out = subprocess.run(cmd, capture_output=True, text=True, timeout=900)
    assert out.returncode == 0, out.stderr[-2000:]
    blocks = [b for b in out.stderr.split("Function Name:")[1:] if kernel in b.split("\n")[0]]
    assert len(blocks) == count, "kernels not found in the resource remarks"
    large = 0
    for b in blocks:
        get = lambda key: int(re.search(key + r":\s*(\d+)", b).group(1))
        assert get("VGPRs Spill") == 0 and get(r"ScratchSize \[bytes/lane\]") == 0, b
        # template arguments: types, rows and columns of the block
        if re.search(r"ILi\dELi\dELi(256|128)ELi256E", b.split("\n")[0]):
            large += 1
            assert get(r"Occupancy \[waves/SIMD\]") >= 2, b
    assert large == (11 if kernel == "tiled_kernel" else 0)
