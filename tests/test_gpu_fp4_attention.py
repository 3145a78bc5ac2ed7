"""The cache's operators together, as a program that serves a model calls them: sequences that grow, fork, end and move, over several layers; captured
graphs, several streams, and the stack of layers."""
import numpy as np
import pytest
import torch

from cache_fp4_cases import Sequences, attention_oracle, worst
from oracle import block_scale as bs
from oracle import cache_fp4 as oc
from paper_2511_10909_amd import binding as mm
from paper_2511_10909_amd import fp4_attention as fa

pytestmark = pytest.mark.gpu
TYPE = {torch.bfloat16: mm.BF16, torch.float16: mm.FP16}
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def bits(t):
    return t.detach().contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


class History:
    """Every sequence's keys and values as the cache should hold them, by layer."""

    def __init__(self, cache, heads, dtype, rotary, seed):
        self.cache, self.heads, self.dtype = cache, heads, dtype
        self.rng = np.random.default_rng(seed)
        self.weights = [(1 + 0.2 * self.rng.standard_normal(cache.dim)).astype(np.float32) for _ in range(2)]
        self.rotation = fa.rotation_table(400, rotary) if rotary else None
        w = [torch.from_numpy(x).cuda() for x in self.weights]
        self.attention = fa.Fp4Attention(heads, dtype, *w, rotation=self.rotation, style=mm.ROTATE_PAIRS, window=90)
        self.held = {}

    def step(self, sequences, counts):
        c, d, t = self.cache, self.cache.dim, TYPE[self.dtype]
        batch = c.batch(sequences, counts)
        for layer in range(c.layers):
            width = (self.heads + 2 * c.kv_heads) * d
            x = (self.rng.standard_normal((batch.tokens, width)) * 2).astype(np.float32)
            wide = torch.zeros((batch.tokens + 1, width + 16), dtype=self.dtype, device="cuda")
            wide[:batch.tokens, :width] = torch.from_numpy(x).cuda().to(self.dtype)
            out = torch.full((batch.tokens + 2, self.heads * d), 7.0, dtype=self.dtype, device="cuda")
            self.attention(wide[:, :width], batch, layer, out)
            torch.cuda.synchronize()
            assert (out[batch.tokens:] == 7.0).all()
            self.check(layer, batch, sequences, counts, bs.values_of(bits(wide[:batch.tokens, :width]), t), bs.values_of(bits(out[:batch.tokens]), t))

    def check(self, layer, batch, sequences, counts, x, got):
        c, d, t = self.cache, self.cache.dim, TYPE[self.dtype]
        x = x.reshape(batch.tokens, -1, d)
        rot = np.zeros((0, 16), np.float32) if self.rotation is None else self.rotation.cpu().numpy()
        positions = np.concatenate([np.arange(c.length(s) - n, c.length(s)) for s, n in zip(sequences, counts)])
        args = dict(eps=1e-6, positions=positions, rotation=rot, rotary=rot.shape[1] if self.rotation is not None else 0, style=oc.PAIRS)
        q = oc.norm_rotate(x[:, :self.heads], self.weights[0], **args)
        k = oc.quantize(oc.norm_rotate(x[:, self.heads:self.heads + c.kv_heads], self.weights[1], **args), bs.FLOOR)[2]
        v = oc.quantize(x[:, self.heads + c.kv_heads:].astype(np.float32), bs.FLOOR)[2]
        memory = c.memory[layer].cpu().numpy().reshape(c.pages, c.kv_heads, c.page_tokens // 32, 34 * d)
        at = 0
        for s, n in zip(sequences, counts):
            held = self.held.setdefault((s, layer), [])
            held.extend(zip(k[at:at + n], v[at:at + n]))
            at += n
            gk, gv, there = oc.read(memory, np.array(c.pages_of(s) or [0]), c.page_tokens, c.length(s), d)
            assert there.all() and len(held) == c.length(s)
            if held:
                assert np.array_equal(gk, np.stack([a for a, _ in held])) and np.array_equal(gv, np.stack([b for _, b in held]))
        seqs = Sequences(0, list(counts), [c.length(s) for s in sequences], d, c.kv_heads, c.page_tokens)
        seqs.memory, seqs.table, seqs.columns = memory, batch.table.cpu().numpy(), batch.table.shape[1]
        want, room, _ = attention_oracle(seqs, bs.values_of(bs.bits_of(q, t), t), self.heads, d ** -0.5, 90)
        assert worst(got.reshape(want.shape), want, room, HALF_STEP[self.dtype]) <= 1.0

    def fork(self, s):
        o = self.cache.fork(s)
        for layer in range(self.cache.layers):
            self.held[(o, layer)] = list(self.held.get((s, layer), []))
        return o


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dim,rotary", [(64, 32), (128, 128), (128, 0)])
def test_sequences_that_grow_fork_end_and_move(dtype, dim, rotary):
    cache = fa.Fp4Cache(2, 24, 2, dim, 32)
    h = History(cache, 6, dtype, rotary, dim)
    a, b, c = cache.new(), cache.new(), cache.new()
    h.step([a, b, c], [70, 1, 33])
    for _ in range(2):
        h.step([c, a, b], [1, 1, 1])
    e = h.fork(a)
    h.step([a, e, b], [1, 3, 0])
    cache.free(c)
    f = h.fork(e)
    cache.free(a)
    assert cache.compact() == cache.pages - cache.free_pages()
    h.step([f, e, b], [40, 1, 2])
    g = cache.new()
    h.step([g, f], [130, 1])
    cache.free(e)
    cache.compact()
    h.step([b, g, f], [1, 1, 1])


def test_a_captured_step_replays_as_the_eager_one():
    """Append and attention of single tokens in one graph that counts the lengths on; eager work of another batch between the replays."""
    d, heads, kv, steps = 128, 8, 2, 6
    results = []
    for captured in (False, True):
        torch.manual_seed(3)
        cache = fa.Fp4Cache(1, 150, kv, d, 64)
        cache.memory.zero_()
        layer = fa.Fp4Attention(heads, rotation=fa.rotation_table(9000, d))
        s, other = cache.new(), cache.new()
        inner = (heads + 2 * kv) * d
        prompt = cache.batch([s], 8000)
        big = torch.empty((8000, heads * d), dtype=torch.bfloat16, device="cuda")
        layer(torch.randn(8000, inner, device="cuda").bfloat16(), prompt, 0, big)
        inputs = torch.randn(steps, 1, inner, device="cuda").bfloat16()
        aside = torch.randn(40, inner, device="cuda").bfloat16()
        cache.extend(s, steps)
        cache.extend(other, 40)
        step, by = fa.Batch(cache, [s], [1]), fa.Batch(cache, [other], [40])
        assert mm.attention_fp4_workspace(mm.BF16, max_length=step.max_length, **step.shape(heads)) > 0
        step.lengths.fill_(8001)
        x, out, out2 = inputs[0].clone(), torch.empty((1, heads * d), dtype=torch.bfloat16, device="cuda"), torch.empty((40, heads * d), dtype=torch.bfloat16, device="cuda")

        def once():
            layer(x, step, 0, out)
            step.lengths.add_(1)
        graph = None
        if captured:
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
                once()
            torch.cuda.synchronize()
        got = []
        for i in range(steps):
            x.copy_(inputs[i])
            graph.replay() if captured else once()
            layer(aside, by, 0, out2)
            torch.cuda.synchronize()
            got.append(out.clone())
        results.append((torch.stack(got), out2.clone(), cache.memory[0, list(cache.pages_of(s))].clone(), int(step.lengths[0])))
    for e, c in zip(*results):
        assert torch.equal(e, c) if isinstance(e, torch.Tensor) else e == c


def test_calls_on_two_streams_at_once():
    cache = fa.Fp4Cache(1, 64, 2, 128, 32)
    layer = fa.Fp4Attention(8)
    sets = []
    for n in (1, 90):
        s = cache.new()
        b0 = cache.batch([s], 700)
        x0 = torch.randn(700, 12 * 128, device="cuda").bfloat16()
        layer(x0, b0, 0, torch.empty((700, 1024), dtype=torch.bfloat16, device="cuda"))
        b = cache.batch([s], n)
        sets.append((torch.randn(n, 12 * 128, device="cuda").bfloat16(), b, torch.empty((n, 1024), dtype=torch.bfloat16, device="cuda"), torch.cuda.Stream()))
    want = []
    for x, b, out, _ in sets:
        want.append(layer(x, b, 0, out).clone())
    torch.cuda.synchronize()
    for x, b, out, stream in sets:
        out.zero_()
    torch.cuda.synchronize()
    for _ in range(20):
        for x, b, out, stream in sets:
            with torch.cuda.stream(stream):
                layer(x, b, 0, out)
    torch.cuda.synchronize()
    for (_, _, out, _), w in zip(sets, want):
        assert torch.equal(out, w)


def test_copies_in_a_graph_keep_their_moves():
    memory = torch.randint(0, 256, (2, 9, 4352), dtype=torch.uint8, device="cuda")
    begin, moves = memory.clone(), torch.tensor([[0, 5], [1, 6]], dtype=torch.int32)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        mm.cache_copy_pages(memory, moves, 9, 4352, 2)
    moves.fill_(3)
    for _ in range(3):
        memory.copy_(begin)
        graph.replay()
        torch.cuda.synchronize()
        want = begin.clone()
        want[:, 5], want[:, 6] = begin[:, 0], begin[:, 1]
        assert torch.equal(memory, want)


def test_the_stack_of_layers_runs():
    r = fa.run_stack(layers=2, width=512, heads=8, kv_heads=2, dim=64, prompt=300, generated=5)
    # four bits: elements of E2M1 are off by at most a sixth where nothing saturates, a quarter where the floor rule does, independently of one another
    assert r["finite"] and r["tokens"] == 305 and 0 < r["relative_error"] < 0.25
