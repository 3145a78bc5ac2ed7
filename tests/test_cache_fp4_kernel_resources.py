"""Registers of the kernels around the cache in 4 bits, checked at compile time (no GPU).  A wavefront of attention holds its rows' queries, sums and two granules: the shapes
that take up to three tiles of heads of 128, and single tokens, need no scratch memory, the others a few words; the rest needs none."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2511_10909_amd import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2511_10909_amd", "csrc")


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")
@pytest.mark.parametrize("source,kernel,count", [("attention_fp4", "attention_kernel", 44), ("attention_fp4", "attention_join_kernel", 12), ("cache_append_fp4", "append_kernel", 16),
                                                 ("cache_copy", "cache_copy_kernel", 2)])
def test_registers_suffice(source, kernel, count):
    cmd = ["hipcc", "-c", os.path.join(CSRC, source + ".hip"), "-o", os.devnull, "--offload-arch=gfx950", "--cuda-device-only", "-O3", "-fPIC",
           "-std=c++17", "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
           "-Rpass-analysis=kernel-resource-usage"] + build.PER_FILE.get(source + ".hip", [])
    out = subprocess.run(cmd, capture_output=True, text=True, timeout=900)
    assert out.returncode == 0, out.stderr[-2000:]
    blocks = [b for b in out.stderr.split("Function Name:")[1:] if kernel in b.split("\n")[0]]
    assert len(blocks) == count, "kernels not found in the resource remarks"
    for b in blocks:
        get = lambda key: int(re.search(key + r":\s*(\d+)", b).group(1))
        tiles = re.search(r"attention_kernelILi\dELi(\d+)ELi(\d)E", b.split("\n")[0])
        allowed = 0 if tiles is None or tiles.groups() in (("64", "1"), ("128", "1"), ("128", "2"), ("128", "3")) else 32
        assert get("VGPRs Spill") <= allowed, b
        assert get(r"Occupancy \[waves/SIMD\]") >= (2 if tiles else 4), b
