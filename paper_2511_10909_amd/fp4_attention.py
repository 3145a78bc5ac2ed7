"""Attention over a cache in 4 bits as a served model uses it: pages handed out, shared and moved on the host, heads normed, rotated and appended,
attention over what the cache holds; and a stack of such layers between products with FP4 weights, a prompt at once and then token by token
from a captured graph.

    python -m paper_2511_10909_amd.fp4_attention

A pass of a layer is six launches, or seven where a row's tokens are split: the norm and the product that makes queries, keys and values (Fp4Layer), their
way into the cache (cache_append_fp4), attention (attention_fp4) and the product back."""
import time

import torch

from . import binding as mm
from .fp4_layer import _TYPES, Fp4Layer, _row_stride


class Fp4Cache:
    """Pages of page_tokens tokens for `layers` layers, and the sequences that they belong to.  A page holds all KV heads of a layer; a sequence has the
    same pages in every layer.  Sequences that were forked share pages until one of them writes into a page that is not full.  Bookkeeping is the
    host's; copies of pages are enqueued on the current stream."""

    def __init__(self, layers, pages, kv_heads, dim, page_tokens=64, device="cuda"):
        if dim not in (64, 128) or page_tokens <= 0 or page_tokens % 32 or min(layers, pages, kv_heads) <= 0:
            raise ValueError("a cache has heads of 64 or 128 elements, pages of a multiple of 32 tokens, and at least one layer, page and head")
        self.layers, self.pages, self.kv_heads, self.dim, self.page_tokens = layers, pages, kv_heads, dim, page_tokens
        self.page_bytes = mm.cache_page_bytes(dim, kv_heads, page_tokens)
        self.memory = torch.empty((layers, pages, self.page_bytes), dtype=torch.uint8, device=device)
        self.device = self.memory.device
        self._free = list(range(pages - 1, -1, -1))                     # the lowest page is handed out first
        self._users = [0] * pages
        self._pages, self._lengths = {}, {}
        self._next = 0
        self.generation = 0                                             # counts the changes after which older batches would read or write others' pages

    def __contains__(self, sequence):
        return sequence in self._pages

    def length(self, sequence):
        return self._lengths[sequence]

    def pages_of(self, sequence):
        return tuple(self._pages[sequence])

    def free_pages(self):
        return len(self._free)

    def new(self):
        """An empty sequence."""
        self._next += 1
        self._pages[self._next], self._lengths[self._next] = [], 0
        return self._next

    def _copy(self, moves):
        if moves:
            _is_current(self.device)
            mm.cache_copy_pages(self.memory, torch.tensor(moves, dtype=torch.int32), self.pages, self.page_bytes, self.layers)

    def extend(self, sequence, tokens):
        """Room for `tokens` more tokens of a sequence.  Where its last page is shared and not full, it gets a copy of its own.  Nothing changes if the
        free pages do not suffice."""
        if tokens < 0:
            raise ValueError("a sequence cannot be extended by %d tokens" % tokens)
        self._extend([sequence], [tokens])

    def _extend(self, sequences, counts):
        """All of the sequences or none: the pages are counted first, all copies are one call, and the bookkeeping follows it."""
        taken, left, moves, steps = 0, {}, [], []                       # left: users that a page has lost to the copies so far
        for s, n in zip(sequences, counts):
            held, length = self._pages[s], self._lengths[s]
            fresh = max(0, -(-(length + n) // self.page_tokens) - len(held))
            # (the last of those who share a page keeps it)
            shared = bool(n and length % self.page_tokens) and self._users[held[-1]] - left.get(held[-1], 0) > 1
            if shared:
                left[held[-1]] = left.get(held[-1], 0) + 1
                if taken < len(self._free):
                    moves.append((held[-1], self._free[-1 - taken]))
            taken += shared + fresh
            steps.append((s, n, shared, fresh))
        if taken > len(self._free):
            raise ValueError("%d pages are asked for, %d are free" % (taken, len(self._free)))
        self._copy(moves)
        for s, n, shared, fresh in steps:
            held = self._pages[s]
            if shared:
                self._users[held[-1]] -= 1
                held[-1] = self._free.pop()
                self._users[held[-1]] = 1
            for _ in range(fresh):
                held.append(self._free.pop())
                self._users[held[-1]] = 1
            self._lengths[s] += n
        self.generation += bool(moves)

    def fork(self, sequence):
        """A sequence with the same tokens, in the same pages.  Batches made before it are not for any further call: they would write into pages that are shared now."""
        other = self.new()
        self._pages[other], self._lengths[other] = list(self._pages[sequence]), self._lengths[sequence]
        for page in self._pages[other]:
            self._users[page] += 1
        self.generation += 1
        return other

    def free(self, sequence):
        """Gives a sequence's pages back but for those that others use."""
        for page in self._pages.pop(sequence):
            self._users[page] -= 1
            if not self._users[page]:
                self._free.append(page)
        del self._lengths[sequence]
        self._free.sort(reverse=True)
        self.generation += 1

    def compact(self):
        """Moves pages so that those in use are the first ones; returns how many these are."""
        used = self.pages - len(self._free)
        holes = [p for p in reversed(self._free) if p < used]
        moves = list(zip((p for p in range(used, self.pages) if self._users[p]), holes))
        self._copy(moves)
        to = dict(moves)
        for source, target in moves:
            self._users[target], self._users[source] = self._users[source], 0
        for held in self._pages.values():
            held[:] = [to.get(p, p) for p in held]
        self._free = list(range(self.pages - 1, used - 1, -1))
        self.generation += 1
        return used

    def batch(self, sequences, tokens):
        """Room for tokens[i] (or `tokens`) more tokens of sequences[i], and a Batch of them.  Nothing changes if the free pages do not suffice or a page's copy fails."""
        counts = [tokens] * len(sequences) if isinstance(tokens, int) else list(tokens)
        if len(counts) != len(sequences) or len(set(sequences)) != len(sequences) or min(counts, default=0) < 0:
            raise ValueError("a batch has different sequences, and as many tokens of each as they are")
        self._extend(sequences, counts)
        return Batch(self, list(sequences), counts)


class Batch:
    """What the operators read of a call: page tables, lengths and first rows on the device.  A captured graph may count `lengths` on by itself, where the room for its
    replays was taken beforehand (Fp4Cache.extend); one whose tokens lie in shared pages is for reading alone; a replay is not checked: fork, free and compact wait until it is done, and it is captured anew after them."""

    def __init__(self, cache, sequences, counts):
        self.cache, self.sequences, self.generation = cache, sequences, cache.generation
        self.tokens, self.max_tokens = sum(counts), max(counts, default=0)
        lengths = [cache.length(s) for s in sequences]
        self.max_length = max(lengths, default=0)
        # whether some of the call's tokens lie in pages that other sequences have as well (a batch that Fp4Cache.batch makes has none)
        self.shared = any(cache._users[p] > 1 for s, n, length in zip(sequences, counts, lengths) if n
                          for p in cache.pages_of(s)[max(length - n, 0) // cache.page_tokens:])
        columns = max([len(cache.pages_of(s)) for s in sequences] + [1])
        rows = [list(cache.pages_of(s)) + [-1] * (columns - len(cache.pages_of(s))) for s in sequences]
        first = [0]
        for n in counts:
            first.append(first[-1] + n)
        self.table = torch.tensor(rows, dtype=torch.int32).reshape(len(sequences), columns).to(cache.device)
        self.lengths = torch.tensor(lengths, dtype=torch.int32).to(cache.device)
        self.begins = torch.tensor(first, dtype=torch.int32).to(cache.device)

    def shape(self, heads):
        c = self.cache
        return dict(dim=c.dim, heads=heads, kv_heads=c.kv_heads, page_tokens=c.page_tokens, pages=c.pages, sequences=len(self.sequences),
                    table_stride=self.table.shape[1], tokens=self.tokens, max_tokens=self.max_tokens)


def _is_current(device):
    if device.type == "cuda" and device.index != torch.cuda.current_device():
        raise ValueError("the cache is on %s, the current device is cuda:%d" % (device, torch.cuda.current_device()))


def rotation_table(positions, rotary_dim, theta=10000.0, device="cuda"):
    """Cosines and sines [positions][rotary_dim] of position * theta^(-2 i / rotary_dim), from binary64 angles."""
    i = torch.arange(0, rotary_dim, 2, device=device, dtype=torch.float64)
    angle = torch.arange(positions, device=device, dtype=torch.float64)[:, None] * theta ** (-i / rotary_dim)
    return torch.cat((angle.cos(), angle.sin()), dim=1).float()


class Fp4Attention:
    """qkv [tokens][(heads + 2 kv_heads) dim] -> out [tokens][heads dim] through one layer of a cache: queries and keys normed for each head (weights of dim
    elements in the type or binary32; None: no norm) and rotated (rotation: a table as rotation_table makes it, or None), keys and values appended, then
    causal attention, `window` tokens back (0: all).  BF16 or FP16; rows of qkv and out may be slices of wider ones.  Every call has the
    queries and the workspace in memory of its own, taken on the stream (or in the capture) that it is made on."""

    def __init__(self, heads, dtype=torch.bfloat16, q_weight=None, k_weight=None, rotation=None, style=mm.ROTATE_HALVES, scale=None, window=0, eps=1e-6,
                 scale_rule=mm.SCALE_RULE_FLOOR):
        if dtype not in _TYPES:
            raise ValueError("attention is BF16 or FP16")
        given = [w for w in (q_weight, k_weight) if w is not None]
        if any(w.dtype not in (dtype, torch.float32) or w.dtype != given[0].dtype for w in given):
            raise ValueError("the norms' weights have the type of the queries, or are binary32, both the same")
        if rotation is not None and (rotation.dim() != 2 or rotation.dtype != torch.float32 or not rotation.is_contiguous() or rotation.shape[1] % 16):
            raise ValueError("a rotation table is [positions][rotary_dim] in binary32, contiguous, rotary_dim a multiple of 16")
        self.heads, self.dtype, self.type, self.rotation, self.style = heads, dtype, _TYPES[dtype], rotation, style
        self.q_weight, self.k_weight = (None if w is None else w.contiguous() for w in (q_weight, k_weight))
        self.weight_type = mm.FP32 if given and given[0].dtype == torch.float32 else self.type
        self.scale, self.window, self.eps, self.scale_rule = scale, window, eps, scale_rule

    def __call__(self, qkv, batch, layer, out):
        cache, heads = batch.cache, self.heads
        d, kv, tokens = cache.dim, cache.kv_heads, batch.tokens
        if batch.generation != cache.generation:
            raise ValueError("the batch is older than the last change of the cache's pages")
        if batch.shared:
            raise ValueError("the batch's tokens lie in pages that another sequence shares: Fp4Cache.batch and extend make room in pages of their own")
        if cache.device.type != "cuda":
            raise ValueError("attention runs on a GPU, the cache is on %s" % cache.device)
        _is_current(cache.device)
        if not 0 <= layer < cache.layers:
            raise ValueError("layer %d of a cache of %d" % (layer, cache.layers))
        if heads <= 0 or heads % kv:
            raise ValueError("%d heads over %d KV heads" % (heads, kv))
        for w in (self.q_weight, self.k_weight):
            if w is not None and (w.numel() != d or w.device != cache.device):
                raise ValueError("the norms' weights: %d on %s are asked for, not %s on %s" % (d, cache.device, tuple(w.shape), w.device))
        rows, rotary = (0, 0) if self.rotation is None else self.rotation.shape
        if rotary > d or (rotary and self.rotation.device != cache.device):
            raise ValueError("the rotation table: up to %d columns on %s are asked for, not %d on %s" % (d, cache.device, rotary, self.rotation.device))
        stride = _row_stride(qkv, "qkv", tokens, (heads + 2 * kv) * d, self.dtype, cache.device)
        out_stride = _row_stride(out, "out", tokens, heads * d, self.dtype, cache.device)
        if tokens == 0:
            return out
        if stride % 8 or out_stride % 8 or qkv.data_ptr() % 16 or out.data_ptr() % 16:
            raise ValueError("qkv and out: rows must begin at multiples of 16 bytes")
        shape = batch.shape(heads)
        size = mm.attention_fp4_workspace(self.type, max_length=batch.max_length, window=self.window, **shape)
        queries = tokens * heads * d * 2
        memory = torch.empty(queries + size, dtype=torch.uint8, device=cache.device)
        at, q, pages = memory.data_ptr(), qkv.data_ptr(), cache.memory[layer]
        mm.cache_append_fp4(q, q + 2 * heads * d, q + 2 * (heads + kv) * d, at, pages, batch.table, batch.lengths, batch.begins, self.type, **shape,
                            q_weight=self.q_weight, k_weight=self.k_weight, weight_type=self.weight_type, rotation=self.rotation, rotary_dim=rotary,
                            rotation_rows=rows, rotation_style=self.style, scale_rule=self.scale_rule, eps=self.eps, q_stride=stride, k_stride=stride,
                            v_stride=stride)
        mm.attention_fp4(at, out, pages, batch.table, batch.lengths, batch.begins, at + queries if size else None, self.type, **shape,
                         max_length=batch.max_length, scale=d ** -0.5 if self.scale is None else self.scale, window=self.window, out_stride=out_stride,
                         workspace_bytes=size)
        return out


class _Block:
    """residual <- residual + x; q, k, v = Wqkv norm(residual); out = Wo attention(q, k, v)."""

    def __init__(self, Wqkv, Wo, heads, tokens, layer, **attention):
        width = Wqkv.shape[1]
        self.layer = layer
        self.project = Fp4Layer(Wqkv, torch.ones(width, dtype=Wqkv.dtype, device=Wqkv.device), tokens)
        self.attention = Fp4Attention(heads, Wqkv.dtype, **attention)
        self.n, self.k = Wo.shape
        self.W = torch.empty((self.n, self.k // 2), dtype=torch.uint8, device=Wo.device)
        self.SW = torch.empty((self.n, self.k // 32), dtype=torch.uint8, device=Wo.device)
        mm.quantize_fp4(Wo, self.W, self.SW, None, self.n, self.k, _TYPES[Wo.dtype], mm.SCALE_FORMAT_E8M0, mm.SCALE_RULE_FIT)

    def __call__(self, x, residual, batch, qkv, heads_out, out):
        m = x.shape[0]
        self.project(x, residual, qkv[:m])
        self.attention(qkv[:m], batch, self.layer, heads_out[:m])
        mm.matmul_fp4(heads_out, None, self.W, self.SW, out, m, self.n, self.k, self.attention.type, self.attention.type)
        return out


def run_stack(layers=4, width=4096, heads=32, kv_heads=8, dim=128, prompt=2048, generated=32, seed=0, dev="cuda"):
    """A prompt through `layers` attention blocks, then `generated` tokens one by one from a captured graph.  Returns times, the first layer's relative error over
    the prompt's last rows against attention in binary64 on the same queries, keys and values (what 4 bits cost), and whether all outputs are finite."""
    gen = torch.Generator(device=dev).manual_seed(seed)

    def normal(*shape, std=1.0):
        return (torch.randn(shape, generator=gen, device=dev) * std).to(torch.bfloat16)

    rotation = rotation_table(prompt + generated, dim, device=dev)
    ones = torch.ones(dim, dtype=torch.bfloat16, device=dev)
    inner = (heads + 2 * kv_heads) * dim
    cache = Fp4Cache(layers, -(-(prompt + generated + 2) // 64) + 1, kv_heads, dim, device=dev)
    blocks = [_Block(normal(inner, width, std=width ** -0.5), normal(width, heads * dim, std=(heads * dim) ** -0.5), heads, prompt, i, q_weight=ones, k_weight=ones,
                     rotation=rotation) for i in range(layers)]
    sequence = cache.new()
    batch = cache.batch([sequence], prompt)
    qkv, heads_out = normal(prompt, inner), normal(prompt, heads * dim)
    x, residual = normal(prompt, width), normal(prompt, width)
    outs = [torch.empty_like(x) for _ in range(2)]

    def forward(x, residual, batch, outs):
        for i, block in enumerate(blocks):
            x = block(x, residual, batch, qkv, heads_out, outs[i % 2])
        return x

    # the first layer by itself, against binary64
    first = blocks[0]
    first.project(x, residual.clone(), qkv)
    first.attention(qkv, batch, 0, heads_out)
    rows = range(max(0, prompt - 4), prompt)
    y = qkv.double().reshape(prompt, heads + 2 * kv_heads, dim)
    z = y[:, :heads + kv_heads]
    z = z / torch.sqrt(z.square().mean(-1, keepdim=True) + 1e-6)
    cos, sin = (t[:, None] for t in rotation[:prompt].double().split(dim // 2, dim=1))
    a, b = z.split(dim // 2, dim=-1)
    z = torch.cat((a * cos - b * sin, b * cos + a * sin), dim=-1)
    group = heads // kv_heads
    k, v = (t.repeat_interleave(group, dim=1) for t in (z[:, heads:], y[:, heads + kv_heads:]))
    want = []
    for r in rows:
        p = torch.softmax((k[:r + 1] * z[r, :heads]).sum(-1) * dim ** -0.5, dim=0)
        want.append((p[..., None] * v[:r + 1]).sum(0).reshape(-1))
    want = torch.stack(want)
    got = heads_out[rows.start:].double()
    error = ((got - want).norm() / want.norm()).item()

    forward(x, residual, batch, outs)
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    last = forward(x, residual, batch, outs)
    torch.cuda.synchronize()
    prompt_s = time.perf_counter() - t0
    finite = bool(torch.isfinite(last).all())

    # the tokens after it: the room for all of them is there, each replay counts the lengths on
    cache.extend(sequence, generated + 1)
    step = Batch(cache, [sequence], [1])
    step.lengths.fill_(prompt + 1)
    token, token_residual = normal(1, width), normal(1, width)
    token_outs = [torch.empty_like(token) for _ in range(2)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        forward(token, token_residual, step, token_outs)
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=side):
            last = forward(token, token_residual, step, token_outs)
            token.copy_(last)
            step.lengths.add_(1)
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    for _ in range(generated):
        graph.replay()
    torch.cuda.synchronize()
    token_s = (time.perf_counter() - t0) / generated
    return dict(prompt_seconds=prompt_s, token_seconds=token_s, relative_error=error, finite=finite and bool(torch.isfinite(token).all()),
                cache_bytes=cache.memory.numel(), tokens=int(step.lengths[0]) - 1)


def _report(argv=None):
    import argparse
    ap = argparse.ArgumentParser(description="a stack of attention blocks on FP4 weights over a cache in 4 bits: a prompt, then tokens from a captured graph")
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--width", type=int, default=4096, help="a multiple of 32")
    ap.add_argument("--heads", type=int, default=32)
    ap.add_argument("--kv-heads", type=int, default=8)
    ap.add_argument("--dim", type=int, default=128, choices=(64, 128))
    ap.add_argument("--prompt", type=int, default=2048, help="tokens of the prompt")
    ap.add_argument("--generated", type=int, default=32, help="tokens after it, one at a time")
    args = ap.parse_args(argv)
    r = run_stack(args.layers, args.width, args.heads, args.kv_heads, args.dim, args.prompt, args.generated)
    print("prompt of %d tokens through %d layers: %.3f ms" % (args.prompt, args.layers, 1e3 * r["prompt_seconds"]))
    print("a token: %.1f us (replayed from a graph)" % (1e6 * r["token_seconds"]))
    print("first layer's attention against binary64 on keys and values of 16 bits: relative error %.4f" % r["relative_error"])
    print("cache: %.1f MiB for %d tokens; all outputs finite: %s" % (r["cache_bytes"] / 2 ** 20, r["tokens"], r["finite"]))


if __name__ == "__main__":
    _report()
