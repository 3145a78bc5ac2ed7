"""The largest sizes that the block-scaled operators take, to the element: decided on the host, no GPU needed."""
import pytest

from paper_2511_10909_amd import binding as mm

P = 1 << 20                                                          # an address that nothing reads: every call here ends before a launch
INVALID, SHAPE = 1, 3


def norm(rows, cols, x_stride=0, residual_stride=0, codes=P):
    mm.rmsnorm_quantize(P, P, None, None, codes, P, rows, cols, mm.BF16, mm.BF16, mm.E4M3, x_stride=x_stride, residual_stride=residual_stride, stream=0)


def quantize(rows, cols, x_stride=0, codes=P):
    mm.quantize_fp4(P, codes, P, None, rows, cols, mm.BF16, x_stride=x_stride, stream=0)


@pytest.mark.parametrize("call,kw", [(norm, {}), (quantize, {}), (norm, dict(x_stride=1 << 25, rows=1 << 23)), (norm, dict(residual_stride=1 << 25, rows=1 << 23)),
                                     (quantize, dict(x_stride=1 << 25, rows=1 << 23)), (norm, dict(rows=1, cols=32, x_stride=1 << 48)), (quantize, dict(rows=1, cols=32, x_stride=1 << 48))])
def test_rows_times_stride_stay_below_2_to_48(call, kw):
    """2^48 elements are refused; one row fewer gets past the sizes (and ends at the next check, a pointer that is missing)."""
    kw = dict(dict(rows=1 << 24, cols=1 << 24), **kw)
    with pytest.raises(mm.MmaemuError) as e:
        call(**kw)
    assert e.value.status == SHAPE
    if kw["rows"] > 1:
        kw["rows"] -= 1
        with pytest.raises(mm.MmaemuError) as e:
            call(**kw, codes=None)
        assert e.value.status == INVALID
