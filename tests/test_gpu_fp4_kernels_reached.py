"""Kernels of the products that only long rows or long loops reach, each asked for by name, and elements that are no numbers."""
import numpy as np
import pytest
import torch

from oracle import block_scale as bs
from paper_2511_10909_amd import binding as mm
from paper_2511_10909_amd import fp4_layer, presets

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


@pytest.mark.parametrize("name,m,n,k", [("blocks of 64 x 64", 250, 4093, 8224), ("blocks of 128 x 128", 500, 8190, 8256)])
def test_long_rows_under_nvfp4_scales(name, m, n, k):
    assert mm.matmul_fp4_kernel(m, n, k, mm.FP16, mm.SCALE_FORMAT_UE4M3) == name
    ops = operands(1, m, n, k, mm.FP16, bs.SCALE_UE4M3)
    check(product(*ops, m, n, k, mm.FP16, bs.SCALE_UE4M3), ops[0], ops[2], ops[3], k, bs.SCALE_UE4M3)


@pytest.mark.parametrize("name,m,n,k", [("stream", 3, 100, 544), ("stream", 16, 9000, 544), ("blocks of 32 x 32", 17, 40, 544), ("blocks of 32 x 64", 77, 5003, 544),
                                        ("blocks of 64 x 64", 250, 4093, 8224), ("blocks of 64 x 128", 250, 8190, 544), ("blocks of 128 x 128", 500, 8190, 8256),
                                        ("blocks of 128 x 256", 250, 28000, 544)])
def test_fp16_both_ways_in_every_kernel(name, m, n, k):
    """Scales of which a tenth leave FP16's range, in both directions."""
    assert mm.matmul_fp4_kernel(m, n, k, mm.FP16) == name
    A, _, W, SW = operands(2, m, n, k, mm.FP16, bs.SCALE_E8M0, 90, 160)
    SW[torch.rand(SW.shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3)) < 0.9] = 120
    check(product(A, None, W, SW, m, n, k, mm.FP16, bs.SCALE_E8M0), A, W, SW, k, bs.SCALE_E8M0)


@pytest.mark.parametrize("k", [2144, 4128])
@pytest.mark.parametrize("code", [mm.E4M3, mm.E5M2])
def test_largest_blocks_over_many_groups_of_scales(code, k):
    """Whole steps over several groups of staged scales, and a step that ends inside: bit for bit the instruction's chain."""
    m, n = 4090, 4085
    assert mm.matmul_fp4_kernel(m, n, k, code) == "blocks of 256 x 256"
    A, SA, W, SW = operands(5, m, n, k, code, bs.SCALE_E8M0)
    assert fp4_layer.model_mismatches(A.view(torch.uint8), SA, W, SW, m, n, k, code) == (0, m * n)


@pytest.mark.parametrize("at,fmt", [(mm.BF16, bs.SCALE_E8M0), (mm.BF16, bs.SCALE_UE4M3), (mm.FP16, bs.SCALE_UE4M3), (mm.FP16, bs.SCALE_E8M0)])
@pytest.mark.parametrize("k", [2144, 4128])
def test_largest_blocks_of_sixteen_bits_over_many_groups_of_scales(k, at, fmt):
    m, n = 4090, 4085
    assert mm.matmul_fp4_kernel(m, n, k, at, fmt) == ("blocks of 128 x 256" if (at, fmt) == (mm.FP16, bs.SCALE_E8M0) else "blocks of 256 x 256")
    A, _, W, SW = operands(6, m, n, k, at, fmt)
    D = product(A, None, W, SW, m, n, k, at, fmt)
    w = weight_values(W, SW, fmt).to(A.dtype)                          # exact
    # 64 products a step: two instructions of 4 x 8 products, 16 apart
    order = np.arange(-(-k // 64) * 64).reshape(-1, 4, 2, 8).transpose(0, 2, 1, 3).reshape(-1)
    order = torch.from_numpy(order[order < k]).cuda()
    Dm, C = (torch.zeros((m, n), dtype=torch.float32, device="cuda") for _ in range(2))
    h = mm.model_create(**presets.GFX950_MFMA[mm.MFMA_F32_16X16X32_BF16 if at == mm.BF16 else mm.MFMA_F32_16X16X32_F16])
    mm.emulate_mma(h, A[:, order].contiguous(), w[:, order].contiguous(), C, Dm, m, n, k, 1, (at, at, mm.FP32, mm.FP32))
    torch.cuda.synchronize()
    mm.model_destroy(h)
    assert torch.equal(D.view(torch.int32), Dm.view(torch.int32))


@pytest.mark.parametrize("code", [mm.E4M3, mm.E5M2])
@pytest.mark.parametrize("m,n,k,slot,waves", [(1, 28672, 8192, 256, 4), (1, 4096, 4096, 256, 8), (3, 3000, 4128, 512, 8), (16, 8192, 2048, 256, 4)])
def test_few_tokens_are_the_models_chains_added_in_order(m, n, k, slot, waves, code):
    """Up to sixteen tokens: each wavefront's slots of the row are one chain of the instruction, their sums are added in binary32 in order.  Nothing
    else comes between the operands and the outputs, and a second call gives the same bits."""
    assert mm.matmul_fp4_kernel(m, n, k, code) == "stream"
    A, SA, W, SW = operands(7, m, n, k, code, bs.SCALE_E8M0)
    A = A.view(torch.uint8)
    D = product(A, SA, W, SW, m, n, k, code, bs.SCALE_E8M0)
    one_a_byte = torch.stack((W & 15, W >> 4), dim=-1).reshape(n, k)
    h = mm.model_create(**presets.GFX950_MFMA[mm.mfma_scale_id(code, mm.E2M1)])
    slots = -(-k // slot)
    total, begin = None, 0
    for wave in range(waves):
        end = min(k, begin + slot * (slots // waves + (wave < slots % waves)))
        C, part = (torch.zeros((m, n), dtype=torch.float32, device="cuda") for _ in range(2))
        if end > begin:
            mm.emulate_mma_scaled(h, A[:, begin:end].contiguous(), one_a_byte[:, begin:end].contiguous(), C, part, SA[:, begin // 32:end // 32].contiguous(),
                                  SW[:, begin // 32:end // 32].contiguous(), 32, m, n, end - begin, 1, (code, mm.E2M1, mm.FP32, mm.FP32))
            torch.cuda.synchronize()
        total = part if total is None else total + part
        begin = end
    mm.model_destroy(h)
    assert begin == k and torch.equal(D, total)
    assert torch.equal(D.view(torch.int32), product(A, SA, W, SW, m, n, k, code, bs.SCALE_E8M0).view(torch.int32))


@pytest.mark.parametrize("m,n,k", [(3, 40, 160), (16, 64, 288), (40, 100, 288), (500, 8190, 544), (250, 28000, 416)])
@pytest.mark.parametrize("code", [mm.E4M3, mm.E5M2])
def test_activation_bytes_that_are_no_numbers(code, m, n, k):
    """A NaN byte makes its token's outputs NaN; an infinity (E5M2) gives infinities of the weights' signs, NaN where the weight is zero and where
    infinities of both signs meet; other tokens are as they were."""
    A, SA, W, SW = operands(8, m, n, k, code, bs.SCALE_E8M0)
    A = A.view(torch.uint8)
    before = product(A, SA, W, SW, m, n, k, code, bs.SCALE_E8M0)
    B = A.clone()
    B[1, k - 3] = 0x7F if code == mm.E4M3 else 0x7E
    if code == mm.E5M2:
        B[m - 1, 33] = 0xFC
        B[0, 5], B[0, 37] = 0x7C, 0x7C
    after = product(B, SA, W, SW, m, n, k, code, bs.SCALE_E8M0)
    assert bool(torch.isnan(after[1]).all())
    touched = [1]
    if code == mm.E5M2:
        touched += [0, m - 1]
        w = weight_values(W, SW, bs.SCALE_E8M0)
        inf, nan = float("inf"), float("nan")
        minus = torch.where(w[:, 33] == 0, nan, -torch.sign(w[:, 33]) * inf)
        two = torch.where(w[:, 5] == 0, nan, torch.sign(w[:, 5]) * inf) + torch.where(w[:, 37] == 0, nan, torch.sign(w[:, 37]) * inf)
        for row, want in ((m - 1, minus), (0, two)):
            assert torch.equal(torch.nan_to_num(after[row].double(), nan=7.0), torch.nan_to_num(want, nan=7.0))
    keep = [i for i in range(m) if i not in touched]
    assert torch.equal(after[keep], before[keep])
