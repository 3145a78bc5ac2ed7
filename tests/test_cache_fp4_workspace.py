"""What attention over a cache in 4 bits takes of workspace, against the bound that a program may rely on (no GPU)."""
import numpy as np

from paper_2511_10909_amd import binding as mm


def test_a_bound_for_every_workspace():
    """A call whose tokens are no more than its sequences' max_tokens never takes more than 268800 rows of dim + 2 numbers; smaller calls may take more than larger ones."""
    rng = np.random.default_rng(0)
    size = lambda **kw: mm.attention_fp4_workspace(mm.BF16, **kw)
    most = 0
    for _ in range(3000):
        log = lambda hi: int(np.exp(rng.uniform(0, np.log(hi))))
        dim, kv, group, sequences, max_tokens = (64, 128)[rng.integers(2)], 2 ** int(rng.integers(0, 5)), log(33), log(300), log(10000)
        s = dict(dim=dim, heads=kv * group, kv_heads=kv, page_tokens=64, pages=10, sequences=sequences, table_stride=10000, tokens=sequences * max_tokens,
                 max_tokens=max_tokens, max_length=max_tokens + log(500000), window=(0, log(20000))[rng.integers(2)])
        if s["max_tokens"] * s["heads"] > 1 << 28:
            continue
        bytes_ = size(**s)
        assert bytes_ <= 268800 * (dim + 2) * 4
        most = max(most, bytes_ / (268800 * (dim + 2) * 4))
    assert most > 0.3
    shape = dict(dim=128, heads=8, kv_heads=8, page_tokens=64, pages=10, sequences=1, table_stride=1000, tokens=3000, max_tokens=3000, max_length=11192)
    assert 0 < size(**shape) < size(window=6000, **shape)
    shape.update(tokens=1, max_tokens=1, max_length=4096)
    assert size(**shape) > size(**dict(shape, sequences=200, tokens=200)) == 0
