"""FP16 activations on MXFP4 weights: what a row's scales change in the columns of its neighbours."""
import numpy as np
import pytest
import torch

from oracle import block_scale as bs
from paper_2511_10909_amd import binding as mm

pytestmark = pytest.mark.gpu


def operands(seed, m, n, k, at, fmt, lo=118, hi=131):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    W = torch.randint(0, 256, (n, k // 2), dtype=torch.uint8, device="cuda", generator=gen)
    SW = torch.randint(*((lo, hi) if fmt == bs.SCALE_E8M0 else (0, 0x7F)), (n, k // (32 if fmt == bs.SCALE_E8M0 else 16)), dtype=torch.uint8, device="cuda", generator=gen)
    x = torch.randn((m, k), device="cuda", generator=gen)
    if at in (mm.BF16, mm.FP16):
        return x.to(torch.bfloat16 if at == mm.BF16 else torch.float16), None, W, SW
    return (x * 16).to(torch.float8_e4m3fn if at == mm.E4M3 else torch.float8_e5m2), torch.randint(120, 128, (m, k // 32), dtype=torch.uint8, device="cuda", generator=gen), W, SW


def weight_values(W, SW, fmt):
    lut = torch.from_numpy(bs.fp4_values(np.arange(16))).cuda()
    unit = torch.exp2(SW.double() - 127) if fmt == bs.SCALE_E8M0 else torch.from_numpy(bs.values_of(np.arange(128, dtype=np.uint8), mm.E4M3)).cuda()[SW.long()]
    return lut[torch.stack((W & 15, W >> 4), dim=-1).reshape(W.shape[0], -1).long()] * unit.repeat_interleave(32 if fmt == bs.SCALE_E8M0 else 16, dim=1)


def product(A, SA, W, SW, m, n, k, at, fmt):
    D = torch.full((m, n), -7.0, device="cuda")
    mm.matmul_fp4(A, SA, W, SW, D, m, n, k, at, mm.FP32, fmt)
    return D


def check(D, A, W, SW, k, fmt):
    w = weight_values(W, SW, fmt)
    want, total = A.double() @ w.t(), A.double().abs() @ w.abs().t()
    # terms cut at 2^-24 of the largest in eight, a sum rounded at 2^-23 for every four products (FP16's second way: two terms a product)
    tol = ((k / 4 + 40) * 2.0 ** -23 + 16 * 2.0 ** -23) * total + want.abs() * 2.0 ** -23
    assert bool(((D.double() - want).abs() <= tol).all())


@pytest.mark.parametrize("m,n,k", [(3, 64, 1024), (16, 64, 1024), (40, 100, 1024), (250, 8190, 544)])
def test_fp16_columns_whose_neighbours_change_ways(m, n, k):
    """One row's scale leaves FP16's range: the kernels then split the activations for its neighbours, too, which sum twice as many terms.  The
    other columns stay within their bound; two calls with the same operands are equal, bit for bit."""
    A, _, W, SW = operands(4, m, n, k, mm.FP16, bs.SCALE_E8M0)
    before = product(A, None, W, SW, m, n, k, mm.FP16, bs.SCALE_E8M0)
    check(before, A, W, SW, k, bs.SCALE_E8M0)
    SW[7, 3] = 150
    after = product(A, None, W, SW, m, n, k, mm.FP16, bs.SCALE_E8M0)
    check(after, A, W, SW, k, bs.SCALE_E8M0)
    assert torch.equal(after, product(A, None, W, SW, m, n, k, mm.FP16, bs.SCALE_E8M0))
    others = torch.arange(n, device="cuda") != 7
    w = weight_values(W, SW, bs.SCALE_E8M0)
    tol = 2 * ((k / 4 + 40) * 2.0 ** -23 + 16 * 2.0 ** -23) * (A.double().abs() @ w.abs().t())
    assert bool(((after - before).double().abs() <= tol)[:, others].all())
