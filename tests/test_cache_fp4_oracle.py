"""The cache's oracle against itself and simple facts (no GPU): where bytes lie, what is written is read, and attention on cases that have a plain answer."""
import numpy as np
import pytest

from oracle import block_scale as bs
from oracle import cache_fp4 as oc
from cache_fp4_cases import Sequences


@pytest.mark.parametrize("d", [64, 128])
def test_every_byte_of_a_granule_has_one_owner(d):
    at = np.concatenate([p.ravel() for p in oc.places(d)])
    assert np.array_equal(np.sort(at), np.arange(34 * d))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [32, 96])
def test_what_is_written_is_read(d, page):
    seqs = Sequences(d + page, [1, 1, 1], [70, 33, 200], d, 3, page)
    held = []
    for s, n in enumerate(seqs.lengths):
        k, v = seqs.heads(n, 3), seqs.heads(n, 3)
        (kc, ks, kv), (vc, vs, vv) = oc.quantize(k, bs.FIT), oc.quantize(v, bs.FLOOR)
        for t in range(n):
            oc.write(seqs.memory, seqs.table[s], page, t, kc[t], ks[t], vc[t], vs[t])
        held.append((kv, vv))
    for s, n in enumerate(seqs.lengths):
        k, v, there = oc.read(seqs.memory, seqs.table[s], page, n, d)
        assert there.all() and np.array_equal(k, held[s][0]) and np.array_equal(v, held[s][1])


def test_scales_stay_within_fp16():
    y = np.zeros((6, 64), dtype=np.float32)
    y[0, 3], y[1, 3], y[2, 3], y[3, 40], y[4, 40] = 1e30, 49152.0, 2.0 ** -30, np.nan, -np.inf
    c, s, v = oc.quantize(y, bs.FIT)
    assert s[0, 0] == 140 and v[0, 3] == 49152.0 and v[1, 3] == 49152.0
    assert (s[5] == 104).all() and s[2, 0] == 104 and v[2, 3] == 0
    assert s[3, 1] == 255 and np.isnan(v[3, 32:]).all() and (v[3, :32] == 0).all() and s[4, 1] == 255
    assert np.array_equal(v[:3].astype(np.float16).astype(np.float64), v[:3])


def test_attention_of_equal_keys_is_a_mean_and_of_one_token_its_value():
    rng = np.random.default_rng(0)
    q, k, v = rng.standard_normal((4, 2, 64)), np.ones((9, 1, 64)), rng.standard_normal((9, 1, 64))
    out = oc.attention(q, k, v, np.ones(9, bool), 5, 0.1, 0)[0]
    for i in range(4):
        assert np.allclose(out[i], v[:6 + i, 0].mean(0))
    out = oc.attention(q, k, v, np.ones(9, bool), 5, 0.1, 1)[0]
    assert np.allclose(out, v[5:, [0, 0]])
    assert (oc.attention(q, k, v, np.ones(9, bool), -4, 0.1, 0)[0] == 0).all()


def test_rotation_keeps_lengths_and_turns_by_the_table():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((3, 2, 64))
    angle = np.array([[0.0, 0.0], [np.pi / 2, 0.0], [np.pi, 1.0]])
    table = np.concatenate([np.cos(angle).repeat(8, 1), np.sin(angle).repeat(8, 1)], 1).astype(np.float32)
    for style in (oc.HALVES, oc.PAIRS):
        y = oc.norm_rotate(x, None, 0.0, np.arange(3), table, 32, style)
        assert np.allclose(np.linalg.norm(y, axis=-1), np.linalg.norm(x, axis=-1), rtol=1e-6) and np.allclose(y[0], x[0], rtol=1e-6)
        a, b = (0, 16) if style == oc.HALVES else (0, 1)
        assert np.allclose(y[1][:, a], -x[1][:, b], atol=1e-6) and np.allclose(y[1][:, b], x[1][:, a], atol=1e-6)
        assert np.allclose(y[..., 32:], x[..., 32:], rtol=1e-6)
    assert np.isnan(oc.norm_rotate(x, None, 0.0, np.array([-1, 0, 3]), table, 32, 0)[[0, 2], :, :32]).all()
