"""Arguments that the block-scaled operators refuse, and calls that are no-ops: decided on the host, no GPU needed."""
import math
import struct

import pytest

from paper_2511_10909_amd import binding as mm

P = 1 << 20                                                          # an address that nothing reads: every call here ends before a launch
INVALID, UNSUPPORTED, SHAPE = 1, 2, 3


def refused(status, fn, *args, **kw):
    with pytest.raises(mm.MmaemuError) as e:
        fn(*args, stream=0, **kw)
    assert e.value.status == status, e.value


def norm_args(**kw):
    a = dict(x=P, residual=P, weight=P, residual_out=P, codes=P, scales=P, rows=2, cols=64, type=mm.BF16, weight_type=mm.BF16, code_type=mm.E4M3)
    a.update(kw)
    return a


@pytest.mark.parametrize("status,kw", [
    (UNSUPPORTED, dict(type=mm.E4M3, weight_type=mm.E4M3)), (UNSUPPORTED, dict(type=mm.FP64, weight_type=mm.FP64)), (UNSUPPORTED, dict(weight_type=mm.FP16)),
    (UNSUPPORTED, dict(code_type=mm.E2M1)), (UNSUPPORTED, dict(code_type=mm.BF16)), (INVALID, dict(scale_rule=2)), (INVALID, dict(eps=-1e-6)),
    (INVALID, dict(eps=math.inf)), (INVALID, dict(eps=math.nan)), (SHAPE, dict(cols=0)), (SHAPE, dict(cols=(1 << 24) + 1)), (SHAPE, dict(x_stride=63)),
    (SHAPE, dict(residual_stride=1)), (SHAPE, dict(rows=1 << 47)), (SHAPE, dict(x_stride=1 << 48)), (INVALID, dict(residual=None)),
    (INVALID, dict(x_stride=65)), (INVALID, dict(x=None, residual_out=None)), (INVALID, dict(codes=None)), (INVALID, dict(scales=None)),
    (INVALID, dict(x=P + 1)), (INVALID, dict(residual=P + 1)), (INVALID, dict(weight=P + 2, weight_type=mm.FP32)), (INVALID, dict(weight=P + 1))])
def test_norm_refuses(status, kw):
    refused(status, mm.rmsnorm_quantize, **norm_args(**kw))


@pytest.mark.parametrize("status,kw", [
    (UNSUPPORTED, dict(type=mm.E5M2)), (INVALID, dict(scale_format=2)), (INVALID, dict(scale_rule=2)), (INVALID, dict(scale_format=1, scale_rule=1)),
    (INVALID, dict(tensor_scale=2.0)), (INVALID, dict(scale_format=1, tensor_scale=0.0)), (INVALID, dict(scale_format=1, tensor_scale=math.inf)),
    (INVALID, dict(scale_format=1, tensor_scale=math.nan)), (SHAPE, dict(cols=0)), (SHAPE, dict(x_stride=31)), (SHAPE, dict(rows=1 << 44)),
    (INVALID, dict(x=None)), (INVALID, dict(codes=None)), (INVALID, dict(scales=None)), (INVALID, dict(x=P + 1)), (INVALID, dict(values=P + 1)),
    (INVALID, dict(values=P, x_stride=65))])
def test_quantize_refuses(status, kw):
    a = dict(x=P, codes=P, scales=P, values=None, rows=2, cols=64, type=mm.BF16)
    a.update(kw)
    refused(status, mm.quantize_fp4, **a)


@pytest.mark.parametrize("status,kw", [
    (UNSUPPORTED, dict(a_type=mm.FP32)), (UNSUPPORTED, dict(a_type=mm.E2M1)), (UNSUPPORTED, dict(d_type=mm.E4M3)), (INVALID, dict(scale_format=2)),
    (UNSUPPORTED, dict(a_type=mm.E4M3, SA=P, scale_format=1)), (INVALID, dict(alpha=math.inf)), (INVALID, dict(alpha=math.nan)), (SHAPE, dict(n=0)),
    (SHAPE, dict(k=0)), (SHAPE, dict(k=48)), (SHAPE, dict(k=(1 << 20) + 32)), (SHAPE, dict(m=(1 << 24) + 1)), (SHAPE, dict(a_stride=56)), (SHAPE, dict(d_stride=4)),
    (SHAPE, dict(d_stride=1 << 39)), (INVALID, dict(A=None)), (INVALID, dict(W=None)), (INVALID, dict(SW=None)), (INVALID, dict(D=None)),
    (INVALID, dict(a_type=mm.E4M3)), (INVALID, dict(SA=P)), (INVALID, dict(A=P + 2)), (INVALID, dict(W=P + 8)), (INVALID, dict(a_stride=68)),
    (INVALID, dict(D=P + 1)), (INVALID, dict(D=P + 2, d_type=mm.FP32))])
def test_product_refuses(status, kw):
    a = dict(A=P, SA=None, W=P, SW=P, D=P, m=3, n=5, k=64, a_type=mm.BF16, d_type=mm.BF16)
    a.update(kw)
    refused(status, mm.matmul_fp4, **a)


def test_no_rows_is_no_work():
    mm.rmsnorm_quantize(None, None, None, None, None, None, 0, 64, mm.BF16, mm.BF16, mm.E4M3, stream=0)
    mm.quantize_fp4(None, None, None, None, 0, 64, mm.BF16, stream=0)
    mm.matmul_fp4(None, None, None, None, None, 0, 8, 64, mm.BF16, mm.BF16, stream=0)


def test_kernel_names_of_products():
    assert mm.matmul_fp4_kernel(1, 4096, 4096, mm.BF16) == "stream" and mm.matmul_fp4_kernel(8192, 8192, 8192, mm.E4M3) == "blocks of 256 x 256"
    for status, args in ((SHAPE, (1, 0, 32, mm.BF16)), (SHAPE, (1, 8, 33, mm.BF16)), (UNSUPPORTED, (1, 8, 32, mm.FP32)), (UNSUPPORTED, (1, 8, 32, mm.E4M3, 1))):
        with pytest.raises(mm.MmaemuError) as e:
            mm.matmul_fp4_kernel(*args)
        assert e.value.status == status


def test_argument_structures():
    """The binding's packed structures are the header's, and one of another size is refused."""
    assert (mm._NORM_ARGS.size, mm._QUANTIZE_ARGS.size, mm._MATMUL_ARGS.size) == (112, 88, 104)
    for fn, packed in ((mm._norm_call, mm._NORM_ARGS), (mm._quantize_call, mm._QUANTIZE_ARGS), (mm._matmul_call, mm._MATMUL_ARGS)):
        assert fn(None) == INVALID
        for size in (0, packed.size - 8, packed.size + 8):
            assert fn(size.to_bytes(4, "little") + bytes(packed.size - 4)) == INVALID


def test_numbers_that_no_argument_holds():
    for kw in (dict(m=1 << 32), dict(n=-1), dict(a_stride=-64), dict(k=64.0)):
        a = dict(A=P, SA=None, W=P, SW=P, D=P, m=3, n=5, k=64, a_type=mm.BF16, d_type=mm.BF16)
        a.update(kw)
        with pytest.raises(struct.error):
            mm.matmul_fp4(**a, stream=0)
    refused(INVALID, mm.matmul_fp4, A=P, SA=None, W=P, SW=P, D=P, m=3, n=5, k=64, a_type=mm.BF16, d_type=mm.BF16, alpha=1e39)
