"""A layer on FP4 weights: slices of wider buffers give what contiguous tensors give, and nothing beside them is written."""
import pytest
import torch

from paper_2511_10909_amd import fp4_layer

pytestmark = pytest.mark.gpu


def normal(*shape, seed=0, dtype=torch.bfloat16):
    return torch.randn(shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).to(dtype)


def slice_of(t, stride, fill=-7.0):
    """t's values as a slice of a wider buffer, and the buffer."""
    wide = torch.full((t.shape[0], stride), fill, dtype=t.dtype, device=t.device)
    wide[:, :t.shape[1]] = t
    return wide[:, :t.shape[1]], wide


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("m", [1, 2, 16, 40])
def test_slices_of_wider_buffers(m, dtype):
    n, k = 200, 320
    layer = fp4_layer.Fp4Layer(normal(n, k, dtype=dtype), normal(k, seed=1, dtype=dtype), 40)
    x, residual = normal(m, k, seed=2, dtype=dtype), normal(m, k, seed=3, dtype=dtype)
    r, out = residual.clone(), torch.empty((m, n), dtype=dtype, device="cuda")
    layer(x, r, out)
    (xs, _), (rs, rw), (os, ow) = slice_of(x, k + 3), slice_of(residual, k + 32), slice_of(torch.zeros_like(out), n + 1)
    layer(xs, rs, os)
    assert torch.equal(os, out) and torch.equal(rs, r)
    assert bool((rw[:, k:] == -7.0).all()) and bool((ow[:, n:] == -7.0).all())
    assert torch.equal(r, (x.float() + residual.float()).to(dtype))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_norm_weights_in_binary32(dtype):
    """Binary32 weights of values that the layer's type holds give what the same values in that type give."""
    n, k, m = 96, 160, 5
    W, w = normal(n, k, dtype=dtype), normal(k, seed=1, dtype=dtype)
    outs = []
    for norm_weight in (w, w.float()):
        x, residual, out = normal(m, k, seed=2, dtype=dtype), normal(m, k, seed=3, dtype=dtype), torch.empty((m, n), dtype=dtype, device="cuda")
        outs.append(fp4_layer.Fp4Layer(W, norm_weight, m)(x, residual, out))
    assert torch.equal(*outs)


def test_a_prompt_on_one_stream_and_tokens_from_a_graph_on_another():
    """Each keeps its own codes: the outputs are those of the same calls one after the other."""
    n = k = 2048
    m, prompts, tokens = 512, 6, 40
    layer = fp4_layer.Fp4Layer(normal(n, k), normal(k, seed=1), m)
    xs = [normal(m, k, seed=10 + i) for i in range(prompts)]
    token, want_token = normal(1, k, seed=5), torch.empty((1, n), dtype=torch.bfloat16, device="cuda")
    layer(token, None, want_token)
    want = [layer(x, None, torch.empty((m, n), dtype=torch.bfloat16, device="cuda")) for x in xs]
    torch.cuda.synchronize()
    one, other, graph = torch.cuda.Stream(), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    token_out, seen = torch.empty_like(want_token), torch.empty((tokens, n), dtype=torch.bfloat16, device="cuda")
    with torch.cuda.graph(graph, stream=other):
        layer(token, None, token_out)
    outs = [torch.empty((m, n), dtype=torch.bfloat16, device="cuda") for _ in xs]
    torch.cuda.synchronize()
    with torch.cuda.stream(one):
        for x, out in zip(xs, outs):
            layer(x, None, out)
    with torch.cuda.stream(other):
        for i in range(tokens):
            graph.replay()
            seen[i].copy_(token_out[0])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    assert torch.equal(seen, want_token.expand_as(seen))
