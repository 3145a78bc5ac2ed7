"""What a layer on FP4 weights passes to the operators and what it refuses: decided on the host, the operators' calls recorded, no GPU needed."""
import pytest
import torch

from paper_2511_10909_amd import fp4_layer

BF16 = torch.bfloat16


@pytest.fixture
def calls(monkeypatch):
    """The operators' calls, by name and position of their arguments."""
    names = {"quantize_fp4": ("x", "codes", "scales", "values", "rows", "cols", "type", "scale_format", "scale_rule", "tensor_scale", "x_stride"),
             "rmsnorm_quantize": ("x", "residual", "weight", "residual_out", "codes", "scales", "rows", "cols", "type", "weight_type", "code_type", "scale_rule", "eps",
                                  "x_stride", "residual_stride"),
             "matmul_fp4": ("A", "SA", "W", "SW", "D", "m", "n", "k", "a_type", "d_type", "scale_format", "alpha", "a_stride", "d_stride")}
    made = []

    def recorded(name):
        def call(*args, **kw):
            made.append((name, dict(zip(names[name], args), **kw)))
        return call

    for name in names:
        monkeypatch.setattr(fp4_layer.mm, name, recorded(name))
    return made


def layer_of(n=48, k=64, tokens=8):
    return fp4_layer.Fp4Layer(torch.zeros((n, k), dtype=BF16), torch.ones(k, dtype=BF16), tokens)


def wide(m, cols, stride):
    return torch.zeros((m, stride), dtype=BF16)[:, :cols]


def test_row_strides_reach_the_operators(calls):
    layer = layer_of()
    x, residual, out = wide(5, 64, 72), wide(5, 64, 100), wide(5, 48, 56)
    del calls[:]
    assert layer(x, residual, out) is out
    (norm, a), (product, b) = calls
    assert (norm, product) == ("rmsnorm_quantize", "matmul_fp4")
    assert a["x"] is x and a["residual"] is residual and a["residual_out"] is residual and b["D"] is out
    assert (a["x_stride"], a["residual_stride"], b.get("d_stride")) == (72, 100, 56)


def test_a_single_row_may_have_any_stride(calls):
    layer = layer_of()
    x, residual, out = (torch.zeros(96, dtype=BF16).as_strided((1, c), (3, 1)) for c in (64, 64, 48))
    del calls[:]
    layer(x, residual, out)
    assert (calls[0][1]["x_stride"], calls[0][1]["residual_stride"], calls[1][1]["d_stride"]) == (64, 64, 48)


@pytest.mark.parametrize("which", [0, 1, 2])
@pytest.mark.parametrize("how", ["every other element", "transposed", "one row for all"])
def test_rows_that_are_not_rows_are_refused(calls, which, how):
    layer = layer_of()
    tensors = [wide(5, c, c) for c in (64, 64, 48)]
    c = tensors[which].shape[1]
    tensors[which] = {"every other element": torch.zeros((5, 2 * c), dtype=BF16)[:, ::2], "transposed": torch.zeros((c, 5), dtype=BF16).t(),
                      "one row for all": torch.zeros((1, c), dtype=BF16).expand(5, c)}[how]
    del calls[:]
    with pytest.raises(ValueError):
        layer(*tensors)
    assert not calls


@pytest.mark.parametrize("which,shape", [(0, (5, 63)), (0, (5, 65)), (0, (5,)), (0, (1, 5, 64)), (0, (9, 64)), (1, (4, 64)), (1, (5, 32)), (1, (64,)), (2, (4, 48)), (2, (5, 47)),
                                         (2, (5, 64)), (2, (48,)), (2, (1, 5, 48))])
def test_other_sizes_are_refused(calls, which, shape):
    """A layer of 64 inputs and 48 outputs for eight tokens: anything else would be read or written beyond its end."""
    layer = layer_of()
    tensors = [torch.zeros(s, dtype=BF16) for s in ((5, 64), (5, 64), (5, 48))]
    tensors[which] = torch.zeros(shape, dtype=BF16)
    del calls[:]
    with pytest.raises(ValueError):
        layer(*tensors)
    assert not calls


@pytest.mark.parametrize("which", [0, 1, 2])
def test_tensors_elsewhere_are_refused(calls, which):
    layer = layer_of()
    tensors = [torch.zeros(s, dtype=BF16) for s in ((5, 64), (5, 64), (5, 48))]
    tensors[which] = tensors[which].to("meta")
    del calls[:]
    with pytest.raises(ValueError):
        layer(*tensors)
    assert not calls


@pytest.mark.parametrize("W,norm_weight", [((64,), (64,)), ((2, 48, 64), (64,)), ((48, 64), (63,)), ((48, 64), (65,)), ((48, 64), (48, 64)), ((0, 64), (64,)), ((48, 0), (0,))])
def test_weights_of_other_sizes_are_refused(calls, W, norm_weight):
    with pytest.raises(ValueError):
        fp4_layer.Fp4Layer(torch.zeros(W, dtype=BF16), torch.zeros(norm_weight, dtype=BF16), 8)
    assert not calls


def test_norm_weights_elsewhere_are_refused(calls):
    with pytest.raises(ValueError):
        fp4_layer.Fp4Layer(torch.zeros((48, 64), dtype=BF16), torch.zeros(64, dtype=BF16, device="meta"), 8)
    assert not calls


def test_a_residual_and_an_output_of_more_rows(calls):
    layer = layer_of()
    residual, out = wide(7, 64, 80), wide(8, 48, 48)
    del calls[:]
    assert layer(wide(5, 64, 64), residual, out) is out
    assert calls[0][1]["rows"] == 5 and calls[0][1]["residual_stride"] == 80 and calls[1][1]["m"] == 5
    del calls[:]
    layer(wide(1, 64, 64), residual, out)
    assert calls[0][1]["rows"] == 1 and calls[1][1]["m"] == 1


def test_no_residual_and_no_tokens(calls):
    layer = fp4_layer.Fp4Layer(torch.zeros((48, 64), dtype=BF16), None, 8)
    del calls[:]
    layer(torch.zeros((3, 64), dtype=BF16), None, torch.zeros((3, 48), dtype=BF16))
    layer(torch.zeros((0, 64), dtype=BF16), torch.zeros((0, 64), dtype=BF16), torch.zeros((0, 48), dtype=BF16))
    assert [(a.get("rows"), a.get("m")) for _, a in calls] == [(3, None), (None, 3), (0, None), (None, 0)]
    assert calls[0][1]["weight"] is None and calls[0][1]["residual"] is None and calls[0][1]["residual_out"] is None


@pytest.mark.parametrize("which", [0, 1, 2])
@pytest.mark.parametrize("dtype", [torch.float16, torch.float32, torch.uint8])
def test_tensors_of_another_type_are_refused(calls, which, dtype):
    layer = layer_of()
    tensors = [torch.zeros(s, dtype=BF16) for s in ((5, 64), (5, 64), (5, 48))]
    tensors[which] = tensors[which].to(dtype)
    del calls[:]
    with pytest.raises(ValueError):
        layer(*tensors)
    assert not calls


@pytest.mark.parametrize("dtype,known", [(BF16, "BF16"), (torch.float16, "FP16")])
def test_norm_weights_in_binary32_or_in_the_layers_type(calls, dtype, known):
    mm = fp4_layer.mm
    for norm_weight, want in ((torch.zeros(64, dtype=dtype), getattr(mm, known)), (torch.zeros(64), mm.FP32), (None, getattr(mm, known))):
        layer = fp4_layer.Fp4Layer(torch.zeros((48, 64), dtype=dtype), norm_weight, 8)
        del calls[:]
        layer(*(torch.zeros(s, dtype=dtype) for s in ((5, 64), (5, 64), (5, 48))))
        assert (calls[0][1]["type"], calls[0][1]["weight_type"]) == (getattr(mm, known), want)
    for other in (torch.float16 if dtype == BF16 else BF16, torch.float64, torch.int16):
        with pytest.raises(ValueError):
            fp4_layer.Fp4Layer(torch.zeros((48, 64), dtype=dtype), torch.zeros(64).to(other), 8)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float64, torch.uint8])
def test_weights_of_other_types_are_refused(calls, dtype):
    with pytest.raises((ValueError, KeyError)):
        fp4_layer.Fp4Layer(torch.zeros((48, 64), dtype=dtype), torch.zeros(64, dtype=dtype), 8)
    assert not calls


@pytest.mark.parametrize("how", ["rows of a wider one", "every other column", "transposed", "one row for all", "one row", "every other row"])
def test_weights_in_any_layout(calls, how):
    """What is quantised are the weights that were given: through the stride of their rows, or as a copy."""
    base = torch.arange(96 * 128).reshape(96, 128).to(BF16)
    W = {"rows of a wider one": base[:, 8:72], "every other column": base[:, ::2], "transposed": base[:64, :48].t(), "one row for all": base[:1, :64].expand(48, 64),
         "one row": base[:, :64].as_strided((1, 64), (5, 1)), "every other row": base[::2, :64]}[how]
    layer = fp4_layer.Fp4Layer(W, None, 8)
    (_, a), = calls
    assert (a["rows"], a["cols"]) == tuple(W.shape) == (layer.n, layer.k)
    seen = torch.as_strided(a["x"], W.shape, (a["x_stride"], 1), a["x"].storage_offset())
    assert a["x_stride"] >= 64 and torch.equal(seen, W)
    if how in ("rows of a wider one", "every other row"):
        assert a["x"] is W                                             # (no copy where the operator takes the layout)


@pytest.mark.parametrize("how", ["every other element", "one for all", "a column"])
def test_norm_weights_in_any_layout(calls, how):
    w = {"every other element": torch.arange(128.0)[::2], "one for all": torch.full((1,), 3.0).expand(64), "a column": torch.arange(128.0).reshape(64, 2)[:, 1]}[how]
    layer = fp4_layer.Fp4Layer(torch.zeros((48, 64), dtype=BF16), w, 8)
    del calls[:]
    layer(*(torch.zeros(s, dtype=BF16) for s in ((5, 64), (5, 64), (5, 48))))
    passed = calls[0][1]["weight"]
    assert passed.is_contiguous() and torch.equal(passed, w)


def test_norm_weights_that_lie_as_the_operator_wants_are_not_copied(calls):
    w = torch.ones(64, dtype=BF16)
    assert fp4_layer.Fp4Layer(torch.zeros((48, 64), dtype=BF16), w, 8).norm_weight is w


def test_calls_share_no_memory(calls, monkeypatch):
    """Two calls' codes and scales lie apart, as calls on two streams need, each within memory taken for its call."""
    layer = layer_of()
    taken = []

    def empty(*args, **kw):
        taken.append(torch.zeros(*args, **{k: v for k, v in kw.items() if k != "device"}))
        return taken[-1]

    monkeypatch.setattr(fp4_layer.torch, "empty", empty)
    del calls[:]
    tokens = 5, 5, 1
    for m in tokens:
        layer(*(torch.zeros(s, dtype=BF16) for s in ((m, 64), (m, 64), (m, 48))))
    assert len(taken) == 3
    for m, memory, (_, a), (_, b) in zip(tokens, taken, calls[0::2], calls[1::2]):
        at = memory.data_ptr()
        codes, scales = a["codes"], a["scales"]
        assert (b["A"], b["SA"]) == (codes, scales) and codes % 16 == 0
        assert at <= codes and codes + 64 * m <= scales and scales + 2 * m <= at + memory.numel() * memory.element_size()


def test_the_report_says_where_differing_outputs_are_expected():
    same, differ = fp4_layer._model_line(0, 400, "blocks of 256 x 256"), fp4_layer._model_line(7, 400, "blocks of 32 x 64")
    assert "0 of 400" in same and "256 x 256" in same and "chain" not in same
    assert "7 of 400" in differ and "blocks of 32 x 64" in differ and "one chain" in differ and "last bits differ" in differ
