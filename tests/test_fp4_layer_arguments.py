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
