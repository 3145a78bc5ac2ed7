"""FP16 activations on MXFP4 weights of which a few rows have the two largest scales (codes 253 and 254, whose weights pass 2^128): every column,
those rows' and their neighbours', against binary64."""
import numpy as np
import pytest
import torch

from oracle import block_scale as bs
from paper_2511_10909_amd import binding as mm

pytestmark = pytest.mark.gpu

SIZES = [("stream", 2, 16, 64), ("stream", 3, 40, 288), ("stream", 8, 100, 1056), ("stream", 16, 4100, 512), ("stream", 13, 17000, 544), ("blocks of 32 x 32", 17, 40, 544),
         ("blocks of 32 x 32", 40, 100, 96), ("blocks of 32 x 64", 77, 5003, 544), ("blocks of 64 x 64", 250, 4093, 8224), ("blocks of 64 x 128", 250, 8190, 544),
         ("blocks of 128 x 128", 500, 8190, 8256), ("blocks of 128 x 256", 250, 28000, 544)]


def weight_values(W, SW):
    lut = torch.from_numpy(bs.fp4_values(np.arange(16))).cuda()
    unit = torch.exp2(SW.double() - 127)
    return lut[torch.stack((W & 15, W >> 4), dim=-1).reshape(W.shape[0], -1).long()] * unit.repeat_interleave(32, dim=1)


@pytest.mark.parametrize("spread", ["one element", "all elements"])
@pytest.mark.parametrize("name,m,n,k", SIZES)
def test_rows_of_the_largest_scales_among_others(name, m, n, k, spread):
    """One row of every sixteen has blocks of codes 253 and 254, at places of its own; with one element in such a block activations are of
    ordinary size and another row in sixteen has the smallest codes, with all elements activations are small."""
    assert mm.matmul_fp4_kernel(m, n, k, mm.FP16) == name
    rng = np.random.default_rng(m + n + k)
    W = rng.integers(0, 256, (n, k // 2), dtype=np.uint8)
    SW = rng.integers(118, 131, (n, k // 32), dtype=np.uint8)
    A = np.clip(rng.standard_normal((m, k)), -1.875, 1.875)
    if spread == "one element":
        SW[3::16] = rng.integers(0, 4, SW[3::16].shape)
    else:
        A *= 2.0 ** -11
    for j in range(5, n, 16):
        for code, block in zip((254, 253), rng.permutation(k // 32)[:2]):
            SW[j, block] = code
            if spread == "one element":                                # a half or minus a half
                W[j, 16 * block:16 * block + 16] = 0
                W[j, 16 * block + rng.integers(16)] = rng.choice([0x01, 0x09, 0x10, 0x90])
    A = A.astype(np.float16)
    A[m - 1, 40] = np.inf
    dA, dW, dSW = torch.from_numpy(A).cuda(), torch.from_numpy(W).cuda(), torch.from_numpy(SW).cuda()
    D = torch.empty((m, n), dtype=torch.float32, device="cuda")
    mm.matmul_fp4(dA, None, dW, dSW, D, m, n, k, mm.FP16, mm.FP32)
    w, a = weight_values(dW, dSW), dA[:m - 1].double()
    want, total = a @ w.t(), a.abs() @ w.abs().t()
    # each activation is two terms; terms cut at 2^-24 of the largest in eight, a sum rounded at 2^-23 for every four products; numbers below
    # 2^-126 have steps of 2^-149
    tol = ((k / 4 + 40) * 2.0 ** -23 + 16 * 2.0 ** -23) * total + want.abs() * 2.0 ** -23 + k * 2.0 ** -149
    assert bool((total < 2.0 ** 128).all())
    error = (D[:m - 1].double() - want).abs()
    assert bool((error <= tol).all()), sorted(set((~(error <= tol)).nonzero()[:, 1].tolist()))[:20]
    # an infinite activation: infinities of its weights' signs, NaN where the weight is zero
    last = D[m - 1].double()
    inf = torch.where(w[:, 40] == 0, float("nan"), torch.sign(w[:, 40]) * float("inf"))
    assert torch.equal(torch.nan_to_num(last, nan=7.0), torch.nan_to_num(inf, nan=7.0))


@pytest.mark.parametrize("m,n", [(4, 48), (40, 100)])
def test_every_pair_of_codes_in_one_instruction(m, n):
    """A row of code 254 beside rows of every code that exists, 255 (NaN) among them."""
    rng = np.random.default_rng(n)
    k = 64
    for first in range(0, 256, n - 1):
        W = np.zeros((n, k // 2), dtype=np.uint8)
        W[:, ::5] = rng.integers(1, 8, W[:, ::5].shape) | rng.integers(0, 2, W[:, ::5].shape) << 3
        SW = np.empty((n, k // 32), dtype=np.uint8)
        SW[:] = np.minimum(first + np.arange(n), 255)[:, None]
        SW[n // 2] = 254, 253
        A = (rng.choice([-1.0, 1.0], (m, k)) * 2.0 ** rng.integers(-11, -7, (m, k))).astype(np.float16)
        dA, dW, dSW = torch.from_numpy(A).cuda(), torch.from_numpy(W).cuda(), torch.from_numpy(SW).cuda()
        D = torch.empty((m, n), dtype=torch.float32, device="cuda")
        mm.matmul_fp4(dA, None, dW, dSW, D, m, n, k, mm.FP16, mm.FP32)
        w = weight_values(dW, dSW)
        nan = (dSW == 255).any(dim=1)
        want, total = dA.double() @ w.t(), dA.double().abs() @ w.abs().t()
        assert bool(torch.isnan(D[:, nan]).all())
        error, tol = (D.double() - want).abs(), (56 + 16) * 2.0 ** -23 * total + want.abs() * 2.0 ** -23 + k * 2.0 ** -149
        assert bool((error <= tol)[:, ~nan].all()), (first, (~(error <= tol)[:, ~nan]).nonzero()[:8].tolist())
