"""Up to sixteen tokens on more weight rows than the units take at once: short and long rows, on either side of what the shapes of the workgroups are chosen by."""
import numpy as np
import pytest
import torch

from oracle import block_scale as bs
from paper_2511_10909_amd import binding as mm

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("at,fmt", [(mm.BF16, bs.SCALE_E8M0), (mm.BF16, bs.SCALE_UE4M3), (mm.FP16, bs.SCALE_E8M0), (mm.FP16, bs.SCALE_UE4M3), (mm.E4M3, bs.SCALE_E8M0), (mm.E5M2, bs.SCALE_E8M0)])
@pytest.mark.parametrize("m,n,k", [(6, 20479, 6144), (8, 20481, 2048), (5, 20481, 2080), (7, 66001, 544), (8, 41003, 4128), (14, 16385, 6144), (9, 16385, 6176), (16, 24576, 1056),
                                   (12, 24577, 2048), (10, 24577, 2080), (14, 25001, 6176), (16, 41003, 2144), (13, 131071, 320), (11, 24577, 8224)])
def test_few_tokens_on_many_rows(m, n, k, at, fmt):
    assert mm.matmul_fp4_kernel(m, n, k, at, fmt) == "stream"
    gen = torch.Generator(device="cuda").manual_seed(m + n)
    W = torch.randint(0, 256, (n, k // 2), dtype=torch.uint8, device="cuda", generator=gen)
    b = 32 if fmt == bs.SCALE_E8M0 else 16
    SW = torch.randint(*((118, 131) if b == 32 else (0, 0x7F)), (n, k // b), dtype=torch.uint8, device="cuda", generator=gen)
    x, SA = torch.randn((m, k), device="cuda", generator=gen), None
    if at in (mm.BF16, mm.FP16):
        A = x.to(torch.bfloat16 if at == mm.BF16 else torch.float16)
        av = A.double()
    else:
        A = (x * 16).to(torch.float8_e4m3fn if at == mm.E4M3 else torch.float8_e5m2)
        SA = torch.randint(120, 128, (m, k // 32), dtype=torch.uint8, device="cuda", generator=gen)
        av = A.double() * torch.exp2(SA.double() - 127).repeat_interleave(32, dim=1)
        A = A.view(torch.uint8)
    D = torch.full((m + 1, n), -7.0, device="cuda")
    mm.matmul_fp4(A, SA, W, SW, D, m, n, k, at, mm.FP32, fmt)
    assert bool((D[m] == -7.0).all())
    lut = torch.from_numpy(bs.fp4_values(np.arange(16))).cuda()
    table = torch.from_numpy(bs.values_of(np.arange(128, dtype=np.uint8), mm.E4M3)).cuda()
    for i in range(0, n, 16384):                                       # (the weights in binary64, some rows at a time)
        w, s = W[i:i + 16384], SW[i:i + 16384]
        unit = torch.exp2(s.double() - 127) if b == 32 else table[s.long()]
        wv = lut[torch.stack((w & 15, w >> 4), dim=-1).reshape(w.shape[0], k).long()] * unit.repeat_interleave(b, dim=1)
        want, total = av @ wv.t(), av.abs() @ wv.abs().t()
        # terms cut at 2^-24 (8-bit activations: 2^-13) of the largest in eight, a sum rounded at 2^-23 for every four products
        tol = ((k / 4 + 40) * 2.0 ** -23 + (16 * 2.0 ** -23 if SA is None else 8 * 2.0 ** -13)) * total + want.abs() * 2.0 ** -23
        assert bool(((D[:m, i:i + 16384].double() - want).abs() <= tol).all()), i
