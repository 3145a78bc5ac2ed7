"""Products with FP4 weights, bit for bit against the emulated instructions that form their sums, and the stack of layers that uses them."""
import numpy as np
import pytest
import torch

from oracle import block_scale as bs
from paper_2511_10909_amd import binding as mm
from paper_2511_10909_amd import fp4_layer, presets

pytestmark = pytest.mark.gpu


def dev(a, shape=None):
    t = torch.from_numpy(np.ascontiguousarray(a).view(np.uint8).copy()).cuda()
    return t if shape is None else t.reshape(shape)


def weights_of(rng, n, k, fmt):
    W = rng.integers(0, 256, (n, k // 2), dtype=np.uint8)
    SW = rng.integers(118, 131, (n, k // 32), dtype=np.uint8) if fmt == bs.SCALE_E8M0 else rng.integers(0, 0x7F, (n, k // 16), dtype=np.uint8)
    return W, SW


# (kernels whose wavefronts split no sum: the first with few products, the others with any number)
@pytest.mark.parametrize("code", [mm.E4M3, mm.E5M2])
@pytest.mark.parametrize("m,n,k,name", [(1, 70, 128, "stream"), (13, 200, 128, "stream"), (16, 5000, 128, "stream"), (40, 100, 96, "blocks of 32 x 32"),
                                        (250, 4093, 128, "blocks of 64 x 64"), (250, 28000, 416, "blocks of 128 x 256"), (4090, 4085, 544, "blocks of 256 x 256"),
                                        (500, 16001, 4128, "blocks of 128 x 256")])
def test_bytes_are_the_models_chain(m, n, k, name, code):
    assert mm.matmul_fp4_kernel(m, n, k, code) == name
    rng = np.random.default_rng(m + n + k)
    A, SA = bs.quantize8(rng.standard_normal((m, k)) * np.exp2(rng.integers(-2, 3, (m, 1))), code, bs.FLOOR)
    W, SW = weights_of(rng, n, k, bs.SCALE_E8M0)
    assert fp4_layer.model_mismatches(dev(A), dev(SA), dev(W), dev(SW), m, n, k, code) == (0, m * n)


@pytest.mark.parametrize("at,fmt", [(mm.BF16, bs.SCALE_E8M0), (mm.BF16, bs.SCALE_UE4M3), (mm.FP16, bs.SCALE_E8M0), (mm.FP16, bs.SCALE_UE4M3)])
@pytest.mark.parametrize("m,n,k", [(1, 70, 128), (7, 100, 128), (16, 200, 128), (16, 20000, 128), (250, 28000, 320), (4090, 4085, 544)])
def test_sixteen_bits_are_the_models_chain(m, n, k, at, fmt):
    """The weights in the activations' type, the products in the order in which the kernels take them."""
    name = mm.matmul_fp4_kernel(m, n, k, at, fmt)
    assert name in ("stream", "blocks of 128 x 256", "blocks of 256 x 256")
    rng = np.random.default_rng(m + n + k)
    A = bs.bits_of((rng.standard_normal((m, k)) * np.exp2(rng.integers(-3, 4, (m, k)))).astype(np.float32), at)
    W, SW = weights_of(rng, n, k, fmt)
    wv = bs.weights(W, SW, fmt)
    wb = bs.bits_of(wv.astype(np.float32), at)
    assert np.array_equal(bs.values_of(wb, at), wv)                    # exact
    # 128 products: four instructions of 4 x 8 products, 32 apart; blocks: 64 products, two instructions of 4 x 8, 16 apart
    part, per = (128, 4) if name == "stream" else (64, 2)
    order = np.arange(-(-k // part) * part).reshape(-1, 4, per, 8).transpose(0, 2, 1, 3).reshape(-1)
    order = order[order < k]                                           # (groups of eight: products beyond the row are whole groups of zeros)
    D, Dm, C = (torch.zeros((m, n), dtype=torch.float32, device="cuda") for _ in range(3))
    mm.matmul_fp4(dev(A), None, dev(W), dev(SW), D, m, n, k, at, mm.FP32, fmt)
    h = mm.model_create(**presets.GFX950_MFMA[mm.MFMA_F32_16X16X32_BF16 if at == mm.BF16 else mm.MFMA_F32_16X16X32_F16])
    mm.emulate_mma(h, dev(A[:, order]), dev(wb[:, order]), C, Dm, m, n, k, 1, (at, at, mm.FP32, mm.FP32))
    torch.cuda.synchronize()
    mm.model_destroy(h)
    assert torch.equal(D.view(torch.int32), Dm.view(torch.int32))


def test_stack_of_layers():
    r = fp4_layer.run_stack(layers=2, width=1024, prompt=100, generated=3)
    assert r["finite"] and r["compared"] == 100 * 1024
    # weights of a normal distribution in blocks of 32: steps of 1/2, 1 and 2 in 6 give an error of about a ninth of their size, the codes'
    # steps of 1/8 .. 1/16 a few hundredths, and nothing else comes near
    assert 0.05 < r["relative_error"] < 0.2


def test_layer_refusals():
    W, one = torch.zeros((64, 96), dtype=torch.bfloat16, device="cuda"), torch.ones(96, dtype=torch.bfloat16, device="cuda")
    layer = fp4_layer.Fp4Layer(W, one, 4)
    x = torch.zeros((5, 96), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError):
        layer(x, x.clone(), torch.empty((5, 64), dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(ValueError):
        fp4_layer.Fp4Layer(W[:, :40].contiguous(), one[:40], 4)


@pytest.mark.parametrize("at,fmt", [(mm.BF16, bs.SCALE_E8M0), (mm.BF16, bs.SCALE_UE4M3), (mm.FP16, bs.SCALE_E8M0), (mm.E4M3, bs.SCALE_E8M0), (mm.E5M2, bs.SCALE_E8M0)])
@pytest.mark.parametrize("m,n,k", [(99, 16841, 3264), (793, 5029, 1632), (1782, 2311, 1632), (210, 17519, 2528), (2328, 1773, 2560), (615, 13097, 1376), (519, 14883, 1696),
                                   (940, 17038, 1280), (2633, 6347, 1312), (250, 4093, 8224), (500, 8190, 8256),
                                   (3, 3000, 8224), (2, 2048, 4096), (4, 6001, 4128), (1, 9001, 1024), (6, 600, 4128), (8, 4096, 2048), (7, 8200, 6304), (5, 8000, 1024), (7, 21000, 608),
                                   (6, 16500, 6016), (14, 1000, 4160), (9, 8192, 3840), (14, 5003, 4384), (10, 9001, 1024), (12, 17000, 1056), (14, 25000, 2144), (16, 28672, 544)])
def test_sizes_around_the_choices_of_kernels(m, n, k, at, fmt):
    """A few tokens or weight rows more than whole rounds of blocks, some of them computed in two parts; few tokens on few and many weight rows
    of whole and broken lines.  Every output against binary64, with strided activations and outputs."""
    if m >= 250 and k > 8192:                                                       # (and the blocks that 16-bit activations take for long rows only)
        assert mm.matmul_fp4_kernel(m, n, k, at, fmt) == ("blocks of 64 x 64" if m == 250 else "blocks of 128 x 128")
    gen = torch.Generator(device="cuda").manual_seed(m + n)
    W = torch.randint(0, 256, (n, k // 2), dtype=torch.uint8, device="cuda", generator=gen)
    b = 32 if fmt == bs.SCALE_E8M0 else 16
    SW = torch.randint(*((118, 131) if b == 32 else (0, 0x7F)), (n, k // b), dtype=torch.uint8, device="cuda", generator=gen)
    lut = torch.from_numpy(bs.fp4_values(np.arange(16))).cuda()
    unit = torch.exp2(SW.double() - 127) if b == 32 else torch.from_numpy(bs.values_of(np.arange(128, dtype=np.uint8), mm.E4M3)).cuda()[SW.long()]
    wv = lut[torch.stack((W & 15, W >> 4), dim=-1).reshape(n, k).long()] * unit.repeat_interleave(b, dim=1)
    x = torch.randn((m, k), device="cuda", generator=gen)
    SA = None
    if at in (mm.BF16, mm.FP16):
        a = x.to(torch.bfloat16 if at == mm.BF16 else torch.float16)
        av = a.double()
        wide = torch.zeros((m, k + 8), dtype=a.dtype, device="cuda")
    else:
        a = (x * 16).to(torch.float8_e4m3fn if at == mm.E4M3 else torch.float8_e5m2)
        SA = torch.randint(120, 128, (m, k // 32), dtype=torch.uint8, device="cuda", generator=gen)
        av = a.double() * torch.exp2(SA.double() - 127).repeat_interleave(32, dim=1)
        a = a.view(torch.uint8)
        wide = torch.zeros((m, k + 16), dtype=a.dtype, device="cuda")
    wide[:, :k] = a
    D = torch.full((m, n + 3), -7.0, device="cuda")
    mm.matmul_fp4(wide, SA, W, SW, D, m, n, k, at, mm.FP32, fmt, 1.0, wide.shape[1], n + 3)
    want, total = av @ wv.t(), av.abs() @ wv.abs().t()
    # terms cut at 2^-24 (8-bit activations: 2^-13) of the largest in eight, a sum rounded at 2^-23 for every four products (twice as many for FP16's second way)
    tol = ((k / 4 + 40) * 2.0 ** -23 + (16 * 2.0 ** -23 if SA is None else 8 * 2.0 ** -13)) * total + want.abs() * 2.0 ** -23
    assert bool(((D[:, :n].double() - want).abs() <= tol).all())
    assert bool((D[:, n:] == -7.0).all())
