"""Appending to a cache in 4 bits where a wavefront takes several heads one after another: as many as the host's bounds of a call make worth it."""
import pytest

from cache_fp4_cases import Sequences
from oracle import block_scale as bs
from paper_2511_10909_amd import binding as mm
from test_gpu_cache_fp4 import inputs, run_append, weights

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("heads,kv", [(5, 3), (9, 2), (11, 5), (16, 8), (3, 9)])
@pytest.mark.parametrize("per", [2, 8])
@pytest.mark.parametrize("parts", ["qkv", "q", "kv"])
def test_append_of_several_heads_a_wavefront(d, heads, kv, per, parts):
    """Bit for bit, with numbers of heads that are no multiples of a wavefront's, tokens that begin anywhere.  max_tokens, a bound, makes the call a large one: two heads a
    wavefront from 8192 on, eight from 65536."""
    seqs = Sequences(d + heads, [13, 0, 1, 6, 29], [70, 40, 33, 6, 61], d, kv, 64)
    groups, read = 4 if d == 128 else 8, (heads if "q" in parts else 0) + (2 * kv if "k" in parts else 0)
    most = {2: 8192, 8: 65536}[per] * groups // (read * len(seqs.fresh)) + groups
    assert {2: 8192, 8: 65536}[per] <= ((most + groups - 2) // groups + 1) * read * len(seqs.fresh) < {2: 16384, 8: 131072}[per]
    for t, wt, rotary, style, rule in ((mm.BF16, mm.BF16, d, mm.ROTATE_HALVES, bs.FLOOR), (mm.FP16, mm.FP32, 32, mm.ROTATE_PAIRS, bs.FIT)):
        qw, kw = weights(seqs, wt)
        x = inputs(seqs, heads, t)
        run_append(seqs, heads, t, x, qw, kw, weight_type=wt, rotary=rotary, style=style, rule=rule, parts=parts, max_tokens=most)
        run_append(seqs, heads, t, x, None, None, rule=rule, parts=parts, pad=8, in_place="q" in parts, max_tokens=most)
