"""quantize_fp4's BF16 values under small tensor scales: below binary32's least normal number, too, they are rounded once."""
import numpy as np
import pytest

import torch

from oracle import block_scale as bs
from paper_2511_10909_amd import binding as mm

pytestmark = pytest.mark.gpu


def bf16_once(v):
    """Binary64 values rounded to BF16's numbers, nearest even (its steps below 2^-126 are 2^-133)."""
    _, e = np.frexp(v)
    step = np.ldexp(1.0, np.maximum(e - 1, -126) - 7)
    return np.rint(v / step) * step


def values(x, ts):
    """x: BF16 patterns.  (values on the GPU, in binary64; the same from the definition, before their rounding)."""
    rows, cols = x.shape
    k = -(-cols // 32) * 32
    dx = torch.from_numpy(x.view(np.int16)).cuda()
    codes = torch.empty((rows, k // 2), dtype=torch.uint8, device="cuda")
    scales = torch.empty((rows, k // 16), dtype=torch.uint8, device="cuda")
    out = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda")
    mm.quantize_fp4(dx, codes, scales, out, rows, cols, mm.BF16, mm.SCALE_FORMAT_UE4M3, mm.SCALE_RULE_FLOOR, ts)
    c, s, v = bs.quantize_fp4(bs.values_of(x, mm.BF16), bs.SCALE_UE4M3, bs.FLOOR, ts)
    assert np.array_equal(codes.cpu().numpy(), c) and np.array_equal(scales.cpu().numpy(), s)
    return out.double().cpu().numpy(), v


def check_once(x, ts):
    got, v = values(x, ts)
    assert np.array_equal(got, bf16_once(v)), (ts, v[got != bf16_once(v)][:4], got[got != bf16_once(v)][:4])
    return v


def test_a_value_just_above_the_middle_of_two_numbers():
    """Element 3 under group scale 15 2^-9 and tensor scale 12023672 2^-147: above the middle by less than binary32 tells."""
    ts = 12023672 * 2.0 ** -147
    s = 15 * 2.0 ** -9
    x = bs.bits_of(np.array([[6.0, 3.0, -3.0] + [0.0] * 13]) * s * ts, mm.BF16)
    v = check_once(x, ts)
    assert v[0, 1] == 3 * s * ts and 0 < v[0, 1] - np.floor(v[0, 1] * 2.0 ** 133) * 2.0 ** -133 - 2.0 ** -134 < 2.0 ** -150


@pytest.mark.parametrize("seed", range(4))
def test_values_next_to_the_middle(seed):
    """Tensor scales that bring a chosen element next to the middle between two BF16 numbers, on either side."""
    rng = np.random.default_rng(seed)
    near = 0
    for _ in range(40):
        scale = bs.values_of(rng.integers(0x10, 0x70, 1, dtype=np.uint8), bs.E4M3)[0]
        element = rng.choice([0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
        middle = (2 * int(rng.integers(1, 127)) + 1) * 2.0 ** -134
        ts = np.float32(middle / (scale * element))
        ts = float(np.nextafter(ts, np.float32(np.inf if rng.random() < 0.5 else 0)))
        x = bs.bits_of(np.array([[6.0, element, -element] + [0.0] * 13]) * scale * ts, mm.BF16)
        v = check_once(x, ts)
        near += bool((np.abs(np.abs(v) - middle) < 2.0 ** -150).any())
    assert near > 4                                                    # (the group's scale comes out as chosen for most of them)


@pytest.mark.parametrize("ts", [2.0 ** -149, 3 * 2.0 ** -149, 2.0 ** -133, 2.0 ** -126, 1.1754942e-38, 1e-36, 2.0 ** -117, 2.0 ** -116, 2.0 ** -115, 1e-30])
def test_values_under_tensor_scales_of_every_size(ts):
    ts = float(np.float32(ts))
    rng = np.random.default_rng(1)
    x = bs.bits_of((rng.standard_normal((64, 96)) * np.exp2(rng.integers(-6, 12, (64, 1))) * ts).astype(np.float32), mm.BF16)
    check_once(x, ts)
