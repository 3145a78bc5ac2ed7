"""The block-scaled operators as a served model uses them: a stack of normed projections on FP4 weights, a prompt at once and
then token by token from a captured graph, and the products' arithmetic held against the emulated instruction.

    python -m paper_2511_10909_amd.fp4_layer

Weights are brought to MXFP4 once (quantize_fp4); a pass of a layer is two launches: the norm with the residual's
addition, whose output leaves as E4M3 codes with E8M0 scales (rmsnorm_quantize), and the product (matmul_fp4)."""
import time

import torch

from . import binding as mm
from . import presets


_TYPES = {torch.bfloat16: mm.BF16, torch.float16: mm.FP16}


def _row_stride(t, what, rows, cols, dtype, device):
    """Elements from one row of t to the next, as the operators count them, for a tensor of at least `rows` rows of `cols` elements."""
    shape = t.shape
    if len(shape) != 2 or shape[0] < rows or shape[1] != cols or t.dtype != dtype or t.device != device:
        raise ValueError("%s: %d rows of %d elements in %s on %s are asked for, not %s in %s on %s" %
                         (what, rows, cols, dtype, device, tuple(shape), t.dtype, t.device))
    apart, step = t.stride()
    if step != 1 and cols > 1:
        raise ValueError("%s: a row's elements must follow one another, not be %d apart" % (what, step))
    if rows <= 1:
        return cols
    if apart < cols:
        raise ValueError("%s: rows of %d elements, %d apart" % (what, cols, apart))
    return apart


class Fp4Layer:
    """x, residual -> W norm(x + residual), residual <- x + residual, for at most `tokens` tokens at a time.  W[n][k] (k a multiple of 32) in BF16 or FP16
    is kept in MXFP4 with scales under which nothing saturates; the norm's weights (None: ones) have W's type or are binary32; both may lie in any
    layout.  x[m][k], the residual (None: no residual stream) and the output have W's type; their rows may be slices of wider ones, and the latter
    two may have more rows than x, which stay as they are.  Every call has its activations' codes and scales in memory of its own, taken on the
    stream (or in the capture) that it is made on: calls on several streams may run at once."""

    def __init__(self, W, norm_weight, tokens, code=mm.E4M3, eps=1e-6):
        if W.dim() != 2 or 0 in W.shape:
            raise ValueError("a layer's weights are W[n][k], not %s" % (tuple(W.shape),))
        self.n, self.k = W.shape
        if self.k % 32:
            raise ValueError("a layer's inputs come in multiples of 32, not %d" % self.k)
        if norm_weight is not None and (norm_weight.numel() != self.k or norm_weight.device != W.device):
            raise ValueError("the norm's weights: %d on %s are asked for, not %s on %s" % (self.k, W.device, tuple(norm_weight.shape), norm_weight.device))
        if W.dtype not in _TYPES or (norm_weight is not None and norm_weight.dtype not in (W.dtype, torch.float32)):
            raise ValueError("a layer's weights are BF16 or FP16, the norm's the same or binary32")
        self.device, self.dtype, self.type = W.device, W.dtype, _TYPES[W.dtype]
        self.norm_type = mm.FP32 if norm_weight is not None and norm_weight.dtype == torch.float32 else self.type
        if (W.stride(1) != 1 and self.k > 1) or (W.stride(0) < self.k and self.n > 1):
            W = W.contiguous()
        self.norm_weight = norm_weight if norm_weight is None else norm_weight.contiguous()
        self.code, self.eps = code, eps
        self.W = torch.empty((self.n, self.k // 2), dtype=torch.uint8, device=W.device)
        self.SW = torch.empty((self.n, self.k // 32), dtype=torch.uint8, device=W.device)
        self.tokens = tokens
        mm.quantize_fp4(W, self.W, self.SW, None, self.n, self.k, self.type, mm.SCALE_FORMAT_E8M0, mm.SCALE_RULE_FIT,
                        x_stride=W.stride(0) if self.n > 1 else self.k)

    def _norm(self, x, residual, m):
        """The codes' memory, m k bytes and m k / 32 of scales after them, with the norm on its way into it."""
        if m > self.tokens:
            raise ValueError("%d tokens in a layer made for %d" % (m, self.tokens))
        k = self.k
        x_stride = _row_stride(x, "x", m, k, self.dtype, self.device)
        residual_stride = 0 if residual is None else _row_stride(residual, "residual", m, k, self.dtype, self.device)
        memory = torch.empty(m * k + m * k // 32, dtype=torch.uint8, device=self.device)
        at = memory.data_ptr()
        mm.rmsnorm_quantize(x, residual, self.norm_weight, residual, at, at + m * k, m, k, self.type, self.norm_type, self.code, mm.SCALE_RULE_FLOOR, self.eps,
                            x_stride, residual_stride)
        return memory

    def activations(self, x, residual):
        """norm(x + residual) as codes [m][k] and scales [m][k / 32]; residual <- x + residual."""
        m = x.shape[0]
        codes, scales = self._norm(x, residual, m).split((m * self.k, m * self.k // 32))
        return codes.view(m, self.k), scales.view(m, self.k // 32)

    def __call__(self, x, residual, out):
        m, k = x.shape[0], self.k
        out_stride = _row_stride(out, "out", m, self.n, self.dtype, self.device)
        memory = self._norm(x, residual, m)
        at = memory.data_ptr()
        mm.matmul_fp4(at, at + m * k, self.W, self.SW, out, m, self.n, k, self.code, self.type, d_stride=out_stride)
        return out


def model_mismatches(A, SA, W, SW, m, n, k, code=mm.E4M3):
    """Outputs of matmul_fp4 (binary32) that differ from the model of v_mfma_scale_f32_16x16x128_f8f6f4 on the same operands, bit for bit, and the
    number of outputs.  The model adds all k products in one chain, as the kernels do whose wavefronts split no sums: those in blocks of
    128 x 256 and 256 x 256, and any kernel for k up to 128.  The others (few tokens, smaller blocks, and the smaller blocks that finish a product in
    two launches) add their wavefronts' chains in binary32, and differ in the last bits."""
    D, Dm, C = (torch.zeros((m, n), dtype=torch.float32, device=A.device) for _ in range(3))
    mm.matmul_fp4(A, SA, W, SW, D, m, n, k, code, mm.FP32)
    one_a_byte = torch.stack((W & 15, W >> 4), dim=-1).reshape(n, k)
    h = mm.model_create(**presets.GFX950_MFMA[mm.mfma_scale_id(code, mm.E2M1)])
    st = torch.empty(mm.STATS_BYTES, dtype=torch.uint8, device=A.device)
    mm.stats_reset(st)
    mm.emulate_mma_scaled(h, A, one_a_byte, C, Dm, SA, SW, 32, m, n, k, 1, (code, mm.E2M1, mm.FP32, mm.FP32))
    mm.compare(D, Dm, m * n, st)
    torch.cuda.synchronize()
    mm.model_destroy(h)
    return mm.read_stats(st)["n_mismatch_bits"], m * n


def run_stack(layers=4, width=4096, prompt=2048, generated=32, seed=0, dev="cuda"):
    """A prompt through `layers` square layers, then `generated` tokens one by one from a captured graph.  Returns times, the first layer's
    relative error against its BF16 weights in binary64 over a few tokens, and model_mismatches of that layer's prompt."""
    gen = torch.Generator(device=dev).manual_seed(seed)

    def normal(*shape, std=1.0):
        return (torch.randn(shape, generator=gen, device=dev) * std).to(torch.bfloat16)

    weights = [normal(width, width, std=width ** -0.5) for _ in range(layers)]
    stack = [Fp4Layer(w, torch.ones(width, dtype=torch.bfloat16, device=dev), prompt) for w in weights]

    def forward(x, residual, outs):
        for i, layer in enumerate(stack):
            x = layer(x, residual, outs[i % 2])
        return x

    x, residual = normal(prompt, width), normal(prompt, width)
    outs = [torch.empty_like(x) for _ in range(2)]
    h = (x[:8].float() + residual[:8].float()).to(torch.bfloat16).double()
    first = stack[0](x, residual.clone(), outs[0])[:8].double()
    want = (h / torch.sqrt(h.square().mean(1, keepdim=True) + 1e-6)) @ weights[0].double().t()
    error = ((first - want).norm() / want.norm()).item()
    mismatches, compared = model_mismatches(*stack[0].activations(x, residual.clone()), stack[0].W, stack[0].SW, prompt, width, width)

    forward(x, residual, outs)
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    forward(x, residual, outs)
    torch.cuda.synchronize()
    prompt_s = time.perf_counter() - t0

    token, token_residual = normal(1, width), normal(1, width)
    token_outs = [torch.empty_like(token) for _ in range(2)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        forward(token, token_residual, token_outs)
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=side):
            last = forward(token, token_residual, token_outs)
            token.copy_(last)
    torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    for _ in range(generated):
        graph.replay()
    torch.cuda.synchronize()
    token_s = (time.perf_counter() - t0) / generated
    return dict(prompt_seconds=prompt_s, prompt_flops=2 * layers * prompt * width * width, token_seconds=token_s, relative_error=error,
                mismatches=mismatches, compared=compared, kernel=mm.matmul_fp4_kernel(prompt, width, width, stack[0].code), finite=bool(torch.isfinite(last).all()))


def _model_line(mismatches, compared, kernel):
    line = "first layer's product (%s) against the model of the scaled instruction: %d of %d outputs differ" % (kernel, mismatches, compared)
    if mismatches:
        line += "; the model adds a row's products in one chain, blocks below 128 x 256 in several: last bits differ there"
    return line


def _report(argv=None):
    import argparse
    ap = argparse.ArgumentParser(description="a stack of normed projections on FP4 weights: a prompt, then tokens from a captured graph")
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--width", type=int, default=4096, help="inputs and outputs of a layer, a multiple of 32")
    ap.add_argument("--prompt", type=int, default=2048, help="tokens of the prompt")
    ap.add_argument("--generated", type=int, default=32, help="tokens after it, one at a time")
    args = ap.parse_args(argv)
    r = run_stack(args.layers, args.width, args.prompt, args.generated)
    print("prompt of %d tokens through %d layers of %d: %.3f ms, %.0f TFLOP/s" % (args.prompt, args.layers, args.width, 1e3 * r["prompt_seconds"],
                                                                                   r["prompt_flops"] / r["prompt_seconds"] / 1e12))
    print("a token: %.1f us (two launches per layer, replayed from a graph)" % (1e6 * r["token_seconds"]))
    print("first layer against its BF16 weights: relative error %.4f" % r["relative_error"])
    print(_model_line(r["mismatches"], r["compared"], r["kernel"]))


if __name__ == "__main__":
    _report()
