"""The binary64 oracle of the block-scaled operators against values worked out by hand and against torch's own float8 types (CPU)."""
import numpy as np
import torch

from oracle import block_scale as bs


def test_fp8_codes_against_torch():
    rng = np.random.default_rng(0)
    v = np.concatenate([rng.standard_normal(20000) * np.exp2(rng.integers(-20, 17, 20000)), [0.0, -0.0, 448, 464, -480, 2.0 ** -10, 3 * 2.0 ** -11]])
    f = v.astype(np.float32)
    for t, tt, top in ((bs.E4M3, torch.float8_e4m3fn, 448.0), (bs.E5M2, torch.float8_e5m2, 57344.0)):
        want = torch.tensor(f).clamp(-top, top).to(tt).view(torch.uint8).numpy()
        assert np.array_equal(bs._codes(f.astype(np.float64), t), want)
        codes = np.arange(256, dtype=np.uint8)
        np.testing.assert_array_equal(bs.values_of(codes, t), torch.tensor(codes).view(tt).double().numpy())


def test_fp4_ties_and_saturation():
    v = np.array([0.25, 0.2500001, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 5.0000001, 7.0, -0.75, -0.0])
    assert list(bs._codes(v, "E2M1")) == [0, 1, 2, 2, 4, 4, 6, 6, 7, 7, 10, 8]


def test_scale_rules():
    a = np.array([448.0, 449.0, 256.0, 511.9, 0.0, 2.0 ** -140, 1.0])
    assert list(bs.e8m0_codes(a, bs.E4M3, bs.FLOOR)) == [127, 127, 127, 127, 0, 0, 119]
    assert list(bs.e8m0_codes(a, bs.E4M3, bs.FIT)) == [127, 128, 127, 128, 0, 0, 119]
    a = np.array([6.0, 6.5, 4.0, 7.9, 3.0])
    assert list(bs.e8m0_codes(a, "E2M1", bs.FLOOR)) == [127, 127, 127, 127, 126]
    assert list(bs.e8m0_codes(a, "E2M1", bs.FIT)) == [127, 128, 127, 128, 126]


def test_groups_that_hold_no_number():
    x = np.zeros((1, 64))
    x[0, 3], x[0, 40] = np.nan, -np.inf
    for fmt, groups, nan in ((bs.SCALE_E8M0, {0, 1}, 0xFF), (bs.SCALE_UE4M3, {0, 2}, 0x7F)):
        c, s, v = bs.quantize_fp4(x, fmt, bs.FLOOR, 1.0)
        assert {i for i in range(s.shape[1]) if s[0, i] == nan} == groups and not c.any() and np.isnan(v[0, 3])


def test_nvfp4_group():
    x = np.zeros((1, 16))
    x[0, :4] = [6.0 * 3.5, 3.5, -7.0, 0.875]                         # group scale 3.5: a UE4M3 number
    c, s, v = bs.quantize_fp4(x, bs.SCALE_UE4M3, bs.FLOOR, 1.0)
    assert bs.values_of(s[:, :1], bs.E4M3) == 3.5 and list(bs.unpack(c)[0, :4]) == [7, 2, 12, 0] and list(v[0, :4]) == [21.0, 3.5, -7.0, 0.0]
    assert c.shape == (1, 16) and s.shape == (1, 2)                  # rows are padded to 32
