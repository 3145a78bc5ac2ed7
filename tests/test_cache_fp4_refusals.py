"""Arguments that the cache's operators refuse, and calls that are no-ops: decided on the host, no GPU needed."""
import math

import pytest
import torch

from paper_2511_10909_amd import binding as mm

P = 1 << 20                                                          # an address that nothing reads: every call here ends before a launch
INVALID, UNSUPPORTED, SHAPE = 1, 2, 3
SIZES = dict(dim=128, heads=8, kv_heads=2, page_tokens=64, pages=10, sequences=2, table_stride=4, tokens=6, max_tokens=3)


def refused(status, fn, *args, **kw):
    with pytest.raises(mm.MmaemuError) as e:
        fn(*args, stream=0, **kw)
    assert e.value.status == status, e.value


SHARED = [
    (UNSUPPORTED, dict(type=mm.FP32)), (UNSUPPORTED, dict(type=mm.E4M3)), (UNSUPPORTED, dict(dim=96)), (UNSUPPORTED, dict(dim=256)), (UNSUPPORTED, dict(dim=0)),
    (SHAPE, dict(page_tokens=0)), (SHAPE, dict(page_tokens=48)), (SHAPE, dict(page_tokens=16)), (SHAPE, dict(page_tokens=65568)), (SHAPE, dict(kv_heads=0)),
    (SHAPE, dict(kv_heads=1025)), (SHAPE, dict(heads=4100)), (SHAPE, dict(pages=0)), (SHAPE, dict(pages=(1 << 30) + 1)), (SHAPE, dict(tokens=(1 << 30) + 1)),
    (SHAPE, dict(max_tokens=(1 << 24) + 1)), (SHAPE, dict(sequences=65536)), (SHAPE, dict(table_stride=0)), (SHAPE, dict(table_stride=1 << 25)),
    (INVALID, dict(cache=None)), (INVALID, dict(table=None)), (INVALID, dict(lengths=None)), (INVALID, dict(begins=None)), (INVALID, dict(cache=P + 8)),
    (INVALID, dict(table=P + 2)), (INVALID, dict(lengths=P + 1)), (INVALID, dict(begins=P + 2)), (SHAPE, dict(q_stride=1016)), (SHAPE, dict(q_stride=1028)),
    (SHAPE, dict(q_stride=(1 << 32) + 8)), (INVALID, dict(q=P + 8))]


@pytest.mark.parametrize("status,kw", SHARED + [
    (UNSUPPORTED, dict(weight_type=mm.FP16)), (UNSUPPORTED, dict(weight_type=mm.E5M2)), (SHAPE, dict(rotary_dim=8)), (SHAPE, dict(rotary_dim=144)),
    (SHAPE, dict(max_tokens=1 << 24, heads=64, kv_heads=8)), (INVALID, dict(rotation_style=2)), (INVALID, dict(scale_rule=2)), (INVALID, dict(eps=-1.0)),
    (INVALID, dict(eps=math.inf)), (INVALID, dict(eps=math.nan)), (SHAPE, dict(k_stride=248)), (SHAPE, dict(v_stride=260)), (SHAPE, dict(q_out_stride=8)),
    (INVALID, dict(q_out=None)), (INVALID, dict(q=None)), (INVALID, dict(q=None, q_out=None)), (INVALID, dict(heads=0)), (INVALID, dict(k=None)), (INVALID, dict(v=None)),
    (INVALID, dict(k=None, v=None, k_values=P)), (INVALID, dict(q_out=P, q_stride=2048)), (INVALID, dict(rotary_dim=64)), (INVALID, dict(rotary_dim=64, rotation=P + 2)),
    (INVALID, dict(k=P + 2)), (INVALID, dict(v=P + 4)), (INVALID, dict(q_out=P + 8)), (INVALID, dict(k_values=P + 8)), (INVALID, dict(v_values=P + 2)),
    (INVALID, dict(q_weight=P + 1)), (INVALID, dict(k_weight=P + 2, weight_type=mm.FP32))])
def test_append_refuses(status, kw):
    a = dict(SIZES, q=P, k=P, v=P, q_out=2 * P, cache=P, table=P, lengths=P, begins=P, type=mm.BF16)
    a.update(kw)
    refused(status, mm.cache_append_fp4, **a)


@pytest.mark.parametrize("status,kw", SHARED + [
    (SHAPE, dict(heads=0)), (SHAPE, dict(heads=7)), (SHAPE, dict(max_tokens=1 << 24)), (SHAPE, dict(max_tokens=1 << 22, heads=1024, kv_heads=1024)),
    (INVALID, dict(scale=0.0)), (INVALID, dict(scale=-1.0)), (INVALID, dict(scale=math.inf)), (INVALID, dict(scale=math.nan)), (INVALID, dict(scale=1e31)),
    (SHAPE, dict(out_stride=1000)), (INVALID, dict(out=P, q_stride=2048)), (INVALID, dict(q=None)), (INVALID, dict(out=None)), (INVALID, dict(out=P + 2)),
    (INVALID, dict(workspace=None)), (INVALID, dict(workspace=P + 8)), (INVALID, dict(workspace_bytes=1 << 10))])
def test_attention_refuses(status, kw):
    a = dict(SIZES, q=P, out=2 * P, cache=P, table=P, lengths=P, begins=P, workspace=P, type=mm.BF16, max_length=100000, scale=0.1, workspace_bytes=1 << 40)
    a.update(kw)
    refused(status, mm.attention_fp4, **a)


def test_workspace_sizes():
    sizes = {k: v for k, v in SIZES.items()}
    assert mm.attention_fp4_workspace(mm.BF16, max_length=32, **sizes) == 0
    big = mm.attention_fp4_workspace(mm.BF16, max_length=100000, **sizes)
    assert big > 0 and big % (6 * 8 * 130 * 4) == 0
    assert mm.attention_fp4_workspace(mm.FP16, max_length=100000, **dict(sizes, sequences=0)) == 0
    assert mm.attention_fp4_workspace(mm.FP16, max_length=100000, window=40, **sizes) < big
    with pytest.raises(mm.MmaemuError) as e:
        mm.attention_fp4_workspace(mm.FP32, max_length=1, **sizes)
    assert e.value.status == UNSUPPORTED
    assert mm._lib.mmaemu_attention_fp4_workspace(bytes(200), None) == INVALID


def moves(*pairs):
    return torch.tensor(pairs, dtype=torch.int32).reshape(-1, 2)


@pytest.mark.parametrize("status,m,kw", [
    (SHAPE, moves((0, 1)), dict(pages=0)), (SHAPE, moves((0, 1)), dict(pages=(1 << 30) + 1)), (SHAPE, moves((0, 1)), dict(page_bytes=0)),
    (SHAPE, moves((0, 1)), dict(page_bytes=24)), (SHAPE, moves((0, 1)), dict(page_bytes=(1 << 32) + 16)), (SHAPE, moves((0, 1)), dict(layers=65536)),
    (SHAPE, moves((0, 1)), dict(layer_bytes=1584)), (SHAPE, moves((0, 1)), dict(layer_bytes=1608)), (SHAPE, moves((0, 1)), dict(layer_bytes=1 << 47)),
    (INVALID, moves((0, 1)), dict(memory=None)), (INVALID, moves((0, 1)), dict(memory=P + 8)), (INVALID, moves((0, 10)), {}), (INVALID, moves((-1, 1)), {}),
    (INVALID, moves((0, 1), (2, 1)), {}), (INVALID, moves((0, 1), (1, 2)), {}), (INVALID, moves((1, 2), (0, 1)), {}), (INVALID, moves((0, 1), (0, 1)), {}),
    (INVALID, moves((0, 1), (1, 0)), {})])
def test_copy_refuses(status, m, kw):
    a = dict(memory=P, pages=10, page_bytes=160, layers=2)
    a.update(kw)
    refused(status, mm.cache_copy_pages, moves=m, **a)


def test_copy_takes_pairs_of_the_host():
    for m in (torch.zeros(2, dtype=torch.int64), torch.zeros(3, dtype=torch.int32), torch.zeros((2, 4), dtype=torch.int32)[:, ::2]):
        with pytest.raises(ValueError):
            mm.cache_copy_pages(P, m, 10, 160, stream=0)


def test_nothing_to_do():
    none = dict(cache=None, table=None, lengths=None, begins=None, type=mm.BF16, stream=0)
    for kw in (dict(sequences=0), dict(tokens=0), dict(max_tokens=0)):
        mm.cache_append_fp4(P, P, P, 2 * P, **none, **dict(SIZES, **kw))
        mm.attention_fp4(None, None, workspace=None, max_length=100, scale=1.0, **none, **dict(SIZES, **kw))
    mm.cache_append_fp4(None, None, None, None, **none, **dict(SIZES, heads=0))
    mm.cache_copy_pages(None, moves(), 10, 160, stream=0)
    mm.cache_copy_pages(None, moves((0, 1)), 10, 160, layers=0, stream=0)


def test_argument_structures():
    for fn, packed in ((mm._append_call, mm._APPEND_ARGS), (mm._attention_call, mm._ATTENTION_ARGS)):
        assert fn(None) == INVALID
        for size in (0, packed.size - 8, packed.size + 8):
            assert fn(size.to_bytes(4, "little") + bytes(packed.size - 4)) == INVALID
