"""Every form of attention over a cache in 4 bits against the binary64 oracle: rows and tokens shared by four and eight wavefronts, one to four tiles of rows, in one part and in several."""
import numpy as np
import pytest

from cache_fp4_cases import Sequences
from cache_fp4_plans import CASES, KV
from paper_2511_10909_amd import binding as mm
from test_gpu_cache_fp4 import run_attention

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("i", range(len(CASES)), ids=["%s, %s x %d%s" % (c["form"], c["fresh"][0], c["group"], ", window %d" % c["window"] if c["window"] else "") for c in CASES])
def test_attention_in_every_form(d, i):
    """Some keys and values are NaN: a token's own in the first sequence, which its last row alone sees, and others' that all rows see, or none within a window.  (The forms' calls
    have the types and sizes of heads by turns.)"""
    c, t = CASES[i], (mm.BF16, mm.FP16)[(i + (d == 64)) % 2]

    def alter(s, k, v):
        if s == 0 and k.shape[0] > 20:
            k[-1, 0, 3], v[-1, 1, 40], v[9, 1, :32] = np.nan, np.inf, np.nan
        if s == 1 and k.shape[0] > 20:
            k[7, 1, d - 1] = np.nan
    seqs = Sequences(d + c["group"] + c["lengths"][0], c["fresh"], c["lengths"], d, KV, 64).fill(alter)
    bounds = dict(c["bounds"])
    longest = bounds.pop("max_length", max(c["lengths"]))
    assert mm.attention_fp4_kernel(t, **dict(seqs.shape(KV * c["group"], **bounds), max_length=longest, window=c["window"])) == c["form"]
    run_attention(seqs, KV * c["group"], t, window=c["window"], pad=8, max_length=longest, **bounds)
