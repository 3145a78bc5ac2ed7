"""The small calls that reach every form of attention over a cache in 4 bits are what they are said to be, and none is missing (no GPU)."""
import re

import pytest

from cache_fp4_plans import CASES, sizes
from paper_2511_10909_amd import binding as mm


@pytest.mark.parametrize("dim", [64, 128])
def test_every_form_is_reached(dim):
    seen = set()
    for c in CASES:
        t, s = sizes(c, dim)
        name = mm.attention_fp4_kernel(t, **s)
        assert name == c["form"]
        parts = int(re.search(r"parts (\d+)", name).group(1))
        rows = mm.attention_fp4_workspace(t, **s)
        assert rows == (parts * s["tokens"] * s["heads"] * (dim + 2) * 4 if parts > 1 else 0)
        seen.add(re.sub(r"parts \d+", "parts" if parts > 1 else "one part", name))
    want = {"tokens over %d wavefronts, tiles %d, %s" % (w, n, p) for w in (4, 8) for n in (1, 2, 3, 4) for p in ("one part", "parts")}
    want |= {"rows over 4 wavefronts, tiles %d, one part%s" % (n, o) for n in (1, 2, 3) for o in ("", ", longest first")}
    want |= {"rows over 4 wavefronts, tiles %d, parts, longest first" % n for n in (1, 2, 3)} | {"rows over 4 wavefronts, tiles 3, parts"}
    assert seen == want


def test_names_of_what_is_refused_or_nothing():
    t, s = sizes(CASES[0], 64)
    assert mm.attention_fp4_kernel(t, **dict(s, tokens=0)) == mm.attention_fp4_kernel(t, **dict(s, sequences=0)) == "none"
    for status, kw in ((3, dict(heads=5)), (2, dict(dim=96)), (3, dict(page_tokens=48))):
        with pytest.raises(mm.MmaemuError) as e:
            mm.attention_fp4_kernel(t, **dict(s, **kw))
        assert e.value.status == status
    assert mm._lib.mmaemu_attention_fp4_kernel(bytes(200), None) == 1 and mm._lib.mmaemu_attention_fp4_kernel(mm._attention_sizes(t, **s), None) == 1
