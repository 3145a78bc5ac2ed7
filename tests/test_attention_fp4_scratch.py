"""Scratch memory of attention over a cache in 4 bits, checked at compile time (no GPU): none where wavefronts have rows of their own, and none in the loop of shapes up to three tiles."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2511_10909_amd import build

SOURCE = os.path.join(build.CSRC, "attention_fp4.hip")


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")
def test_scratch_is_a_few_words_at_most():
    out = subprocess.run(["hipcc", "-c", SOURCE, "-o", os.devnull, "--cuda-device-only", "-Rpass-analysis=kernel-resource-usage"] + build.COMMON, capture_output=True, text=True,
                         timeout=900)
    assert out.returncode == 0, out.stderr[-2000:]
    seen = set()
    for b in out.stderr.split("Function Name:")[1:]:
        shape = re.search(r"attention_kernelILi\dELi(\d+)ELi(\d)ELi(\d)ELi(\d)E", b.split("\n")[0])
        if shape is None:
            continue
        dim, tiles, row_waves, waves = map(int, shape.groups())
        words = int(re.search(r"VGPRs Spill:\s*(\d+)", b).group(1))
        # four tiles, of which no more than drafts have: up to eight words; three tiles of heads of 64 that share tokens: one, read again every 64 granules
        allowed = 0 if row_waves == 4 else 8 if tiles == 4 else 1 if (dim, tiles) == (64, 3) else 0
        assert words <= allowed, (shape.group(0), words)
        seen.add((dim, tiles, row_waves, waves))
    assert seen == {(d, n, 4, 4) for d in (64, 128) for n in (1, 2, 3)} | {(d, n, 1, w) for d in (64, 128) for n in (1, 2, 3, 4) for w in (4, 8)}
