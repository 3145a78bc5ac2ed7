"""Bookkeeping of the cache's pages (no GPU): what is handed out, shared, copied, given back and moved, against a copy of every sequence's tokens."""
import numpy as np
import pytest
import torch

from paper_2511_10909_amd import binding as mm
from paper_2511_10909_amd import fp4_attention as fa


@pytest.fixture
def copies(monkeypatch):
    """Page copies on host memory in place of the library's."""
    calls = []

    def copy(memory, moves, pages, page_bytes, layers=1, layer_bytes=0, stream=None):
        m = moves.tolist()
        assert memory.shape == (layers, pages, page_bytes) and len({t for _, t in m}) == len(m) and not {t for _, t in m} & {s for s, _ in m}
        memory[:, [t for _, t in m]] = memory[:, [s for s, _ in m]].clone()
        calls.append(m)
    monkeypatch.setattr(mm, "cache_copy_pages", copy)
    return calls


class Model:
    """Each token is a number, written into the page's first bytes as the operator would; read back through the tables."""

    def __init__(self, cache, seed):
        self.cache, self.tokens, self.rng, self.count = cache, {}, np.random.default_rng(seed), 0
        cache.memory.zero_()

    def append(self, s, n):
        begin = self.cache.length(s)
        self.cache.extend(s, n)
        for t in range(begin, begin + n):
            self.count = self.count % 250 + 1
            page = self.cache.pages_of(s)[t // self.cache.page_tokens]
            self.cache.memory[:, page, t % self.cache.page_tokens] = self.count
            self.tokens[s].append(self.count)

    def check(self):
        c = self.cache
        users = [0] * c.pages
        for s, want in self.tokens.items():
            assert c.length(s) == len(want) and len(c.pages_of(s)) == -(-len(want) // c.page_tokens)
            for t, x in enumerate(want):
                assert (c.memory[:, c.pages_of(s)[t // c.page_tokens], t % c.page_tokens] == x).all()
            for p in c.pages_of(s):
                users[p] += 1
        assert users == c._users and sorted(c._free) == [p for p in range(c.pages) if not users[p]]


@pytest.mark.parametrize("seed", range(6))
def test_any_order_of_calls_keeps_every_sequence(copies, seed):
    cache = fa.Fp4Cache(2, 20, 1, 64, 32, device="cpu")
    m = Model(cache, seed)
    for _ in range(120):
        what, held = m.rng.integers(0, 10), list(m.tokens)
        if what < 2 or not held:
            m.tokens[cache.new()] = []
        elif what < 6:
            s = held[m.rng.integers(len(held))]
            n = int(m.rng.integers(0, 70))
            before = cache.free_pages(), cache.pages_of(s), cache.length(s)
            try:
                m.append(s, n)
            except ValueError:
                assert (cache.free_pages(), cache.pages_of(s), cache.length(s)) == before
        elif what < 7:
            s = held[m.rng.integers(len(held))]
            m.tokens[cache.fork(s)] = list(m.tokens[s])
        elif what < 9:
            s = held[m.rng.integers(len(held))]
            cache.free(s)
            del m.tokens[s]
        else:
            used = cache.compact()
            assert used == cache.pages - cache.free_pages() and all(p < used for s in m.tokens for p in cache.pages_of(s))
        m.check()


def test_a_fork_copies_a_page_only_when_one_of_two_writes_into_it(copies):
    cache = fa.Fp4Cache(1, 8, 1, 64, 32, device="cpu")
    a = cache.new()
    cache.extend(a, 40)
    b = cache.fork(a)
    assert cache.pages_of(a) == cache.pages_of(b) and not copies
    cache.extend(b, 1)
    assert len(copies) == 1 and cache.pages_of(a)[0] == cache.pages_of(b)[0] and cache.pages_of(a)[1] != cache.pages_of(b)[1]
    cache.extend(a, 1)
    assert len(copies) == 1
    c = cache.fork(a)
    cache.extend(c, 0)
    assert len(copies) == 1 and cache.pages_of(a) == cache.pages_of(c)


def test_a_batch_takes_all_or_nothing(copies):
    cache = fa.Fp4Cache(1, 3, 1, 64, 32, device="cpu")
    a, b = cache.new(), cache.new()
    with pytest.raises(ValueError):
        cache.batch([a, b], [64, 33])
    assert cache.free_pages() == 3 and cache.length(a) == 0
    for wrong in (([a, a], 1), ([a], [1, 2]), ([a], [-1])):
        with pytest.raises(ValueError):
            cache.batch(*wrong)
    batch = cache.batch([b, a], [33, 5])
    assert batch.tokens == 38 and batch.max_tokens == 33 and batch.max_length == 33 and batch.begins.tolist() == [0, 33, 38] and batch.lengths.tolist() == [33, 5]
    assert batch.table.tolist() == [list(cache.pages_of(b)), list(cache.pages_of(a)) + [-1]]
    assert cache.batch([], 1).tokens == 0


def test_refusals():
    for kw in (dict(dim=96), dict(page_tokens=48), dict(page_tokens=0), dict(pages=0), dict(layers=0), dict(kv_heads=0)):
        a = dict(layers=1, pages=2, kv_heads=1, dim=64, page_tokens=32)
        a.update(kw)
        with pytest.raises(ValueError):
            fa.Fp4Cache(device="cpu", **a)
    cache = fa.Fp4Cache(1, 2, 2, 64, 32, device="cpu")
    s = cache.new()
    with pytest.raises(ValueError):
        cache.extend(s, -1)
    with pytest.raises(ValueError):
        fa.Fp4Attention(4, torch.float32)
    with pytest.raises(ValueError):
        fa.Fp4Attention(4, q_weight=torch.ones(64, dtype=torch.float16))
    with pytest.raises(ValueError):
        fa.Fp4Attention(4, q_weight=torch.ones(64), k_weight=torch.ones(64, dtype=torch.bfloat16))
    for table in (torch.ones((4, 24)), torch.ones(16), torch.ones((4, 16), dtype=torch.float64), torch.ones((4, 32))[:, ::2]):
        with pytest.raises(ValueError):
            fa.Fp4Attention(4, rotation=table)
    batch = cache.batch([s], 3)
    good = dict(qkv=torch.zeros((3, 8 * 64), dtype=torch.bfloat16), batch=batch, layer=0, out=torch.zeros((3, 4 * 64), dtype=torch.bfloat16))
    other = lambda **kw: {**good, **kw}
    for layer, kw in ((fa.Fp4Attention(4), other(layer=1)), (fa.Fp4Attention(3), good), (fa.Fp4Attention(4), other(qkv=good["qkv"][:2])),
                      (fa.Fp4Attention(4), other(qkv=good["qkv"].half())), (fa.Fp4Attention(4), other(out=good["out"][:, :64])),
                      (fa.Fp4Attention(4, q_weight=torch.ones(32)), good), (fa.Fp4Attention(4, rotation=torch.ones((9, 128))), good),
                      (fa.Fp4Attention(4), other(qkv=torch.zeros((3, 8 * 64 + 4), dtype=torch.bfloat16)[:, :512])),
                      (fa.Fp4Attention(4), other(out=torch.zeros((4, 4 * 64 + 1), dtype=torch.bfloat16)[:, 1:]))):
        with pytest.raises(ValueError):
            layer(**kw)
    cache.free(s)
    with pytest.raises(ValueError):
        fa.Fp4Attention(4)(**good)


def test_a_batch_older_than_a_fork_is_refused(copies):
    """It would write into pages that two sequences share by then."""
    cache = fa.Fp4Cache(1, 4, 1, 64, 32, device="cpu")
    a = cache.new()
    batch = cache.batch([a], 5)
    cache.fork(a)
    with pytest.raises(ValueError):
        fa.Fp4Attention(1)(torch.zeros((5, 3 * 64), dtype=torch.bfloat16), batch, 0, torch.zeros((5, 64), dtype=torch.bfloat16))


def test_a_copy_that_fails_takes_no_page(monkeypatch):
    def fail(*a, **kw):
        raise RuntimeError("no")
    monkeypatch.setattr(mm, "cache_copy_pages", fail)
    cache = fa.Fp4Cache(1, 4, 1, 64, 32, device="cpu")
    a = cache.new()
    cache.extend(a, 5)
    b = cache.fork(a)
    with pytest.raises(RuntimeError):
        cache.extend(b, 1)
    assert cache.free_pages() == 3 and cache.pages_of(b) == cache.pages_of(a) and cache.length(b) == 5 and cache._users == [2, 0, 0, 0]


def test_work_for_another_device_than_the_current_one_is_refused(copies, monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    cache = fa.Fp4Cache(1, 4, 1, 64, 32, device="cpu")
    a = cache.new()
    batch = cache.batch([a], 5)
    cache.device = torch.device("cuda", 1)
    with pytest.raises(ValueError):
        fa.Fp4Attention(1)(torch.zeros((5, 3 * 64), dtype=torch.bfloat16), batch, 0, torch.zeros((5, 64), dtype=torch.bfloat16))
    b = cache.fork(a)
    with pytest.raises(ValueError):
        cache.extend(b, 1)
    assert not copies
