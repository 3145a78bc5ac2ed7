"""Batches over shared pages (no GPU): one call copies all of them, a batch that cannot be had changes nothing, and shared pages are not written."""
import pytest
import torch

from paper_2511_10909_amd import binding as mm
from paper_2511_10909_amd import fp4_attention as fa


def state(cache):
    return (list(cache._free), list(cache._users), {s: list(p) for s, p in cache._pages.items()}, dict(cache._lengths), cache.generation, cache.memory.clone())


def same(a, b):
    return all(torch.equal(x, y) if isinstance(x, torch.Tensor) else x == y for x, y in zip(a, b))


@pytest.fixture
def copies(monkeypatch):
    """Page copies on host memory in place of the library's; the first `fine` of them succeed."""
    calls = []
    calls_before_failure = [10 ** 9]

    def copy(memory, moves, pages, page_bytes, layers=1, layer_bytes=0, stream=None):
        if len(calls) >= calls_before_failure[0]:
            raise mm.MmaemuError(4, "no")
        m = moves.tolist()
        assert len({t for _, t in m}) == len(m) and not {t for _, t in m} & {s for s, _ in m}
        memory[:, [t for _, t in m]] = memory[:, [s for s, _ in m]].clone()
        calls.append(m)
    monkeypatch.setattr(mm, "cache_copy_pages", copy)
    return calls, calls_before_failure


@pytest.mark.parametrize("with_first", [False, True])
def test_a_batch_of_forks_is_one_copy(copies, with_first):
    """Sixteen forks of a sequence write into its last page at once: whoever is the last to share it keeps it."""
    calls, _ = copies
    cache = fa.Fp4Cache(2, 40, 1, 64, 32, device="cpu")
    cache.memory.copy_(torch.arange(2 * 40).reshape(2, 40, 1).to(torch.uint8).expand_as(cache.memory))
    a = cache.new()
    cache.extend(a, 40)
    first, last = cache.pages_of(a)
    forks = [cache.fork(a) for _ in range(16)]
    batch = cache.batch(forks + [a] * with_first, [1 + i % 3 for i in range(16 + with_first)])
    assert len(calls) == 1 and len(calls[0]) == 16 and {s for s, _ in calls[0]} == {last}
    assert cache.pages_of(a) == (first, last) and cache._users[last] == 1 and cache._users[first] == 17
    own = [cache.pages_of(s)[1] for s in forks]
    assert len(set(own)) == 16 and all(cache._users[p] == 1 for p in own) and (cache.memory[0, own] == last).all() and (cache.memory[1, own] == 40 + last).all()
    assert batch.generation == cache.generation and batch.table[:, 1].tolist() == own + [last] * with_first
    assert [cache.length(s) for s in forks] == [41 + i % 3 for i in range(16)]


def test_a_page_that_only_the_batch_shares_is_counted_as_often_as_it_is_copied(copies):
    """Two sequences share their last page, one page is free: one of them takes it, the other keeps what it has."""
    calls, _ = copies
    cache = fa.Fp4Cache(1, 2, 1, 64, 32, device="cpu")
    a = cache.new()
    cache.extend(a, 5)
    b = cache.fork(a)
    cache.batch([b, a], 1)
    assert len(calls) == 1 and cache.free_pages() == 0 and cache.pages_of(a) != cache.pages_of(b) and cache.length(a) == cache.length(b) == 6


def test_a_copy_that_fails_leaves_every_sequence_as_it_was(copies):
    calls, fails_after = copies
    cache = fa.Fp4Cache(1, 12, 1, 64, 32, device="cpu")
    cache.memory.zero_()
    a, b, c = cache.new(), cache.new(), cache.new()
    cache.extend(a, 5)
    cache.extend(b, 40)
    others = [cache.fork(a), cache.fork(b)]
    for fine in (0, 1):
        fails_after[0] = len(calls) + fine
        before = state(cache)
        if fine == 0:
            with pytest.raises(mm.MmaemuError):
                cache.batch([c, a, b], [70, 1, 1])
            assert same(state(cache), before)
        else:
            cache.batch([c, a, b], [70, 1, 1])
            assert cache.length(c) == 70 and cache.length(a) == 6 and cache.length(b) == 41 and len(set(cache.pages_of(a)) & set(cache.pages_of(others[0]))) == 0


def test_a_batch_without_room_changes_nothing(copies):
    calls, _ = copies
    cache = fa.Fp4Cache(1, 4, 1, 64, 32, device="cpu")
    cache.memory.zero_()
    a = cache.new()
    cache.extend(a, 40)
    b, c = cache.fork(a), cache.new()
    before = state(cache)
    for sequences, counts in (([a, b, c], [1, 1, 60]), ([c, a, b], [33, 1, 1]), ([a, b], [60, 60])):
        with pytest.raises(ValueError):
            cache.batch(sequences, counts)
        assert same(state(cache), before) and not calls
    with pytest.raises(KeyError):
        cache.batch([a, 99], 1)
    assert same(state(cache), before) and not calls


def test_tokens_in_shared_pages_are_not_written(copies):
    """A batch made of a sequence as it is, after a fork: its tokens are the other sequence's as well."""
    cache = fa.Fp4Cache(1, 6, 1, 64, 32, device="cpu")
    a, b = cache.new(), cache.new()
    cache.extend(a, 40)
    cache.extend(b, 64)
    for s in (a, b):
        assert not fa.Batch(cache, [s], [1]).shared
    fork = cache.fork(a)
    x, out = torch.zeros((9, 3 * 64), dtype=torch.bfloat16), torch.zeros((9, 64), dtype=torch.bfloat16)
    for s, n in ((a, 1), (fork, 9)):
        batch = fa.Batch(cache, [b, s], [0, n])
        assert batch.shared
        with pytest.raises(ValueError, match="shares"):
            fa.Fp4Attention(1)(x, batch, 0, out)
    assert not fa.Batch(cache, [a, b], [0, 64]).shared and not cache.batch([a, b], [1, 1]).shared
    # a copy of its own for the last page, the first is shared still
    assert not fa.Batch(cache, [a], [9]).shared and fa.Batch(cache, [a], [10]).shared


def test_a_cache_in_the_hosts_memory_is_not_for_the_gpu(monkeypatch):
    """Its bookkeeping works; no kernel is given its addresses."""
    def reached(*a, **kw):
        raise AssertionError("a kernel's arguments were made")
    for name in ("cache_append_fp4", "attention_fp4", "attention_fp4_workspace"):
        monkeypatch.setattr(mm, name, reached)
    monkeypatch.setattr(mm._lib, "mmaemu_cache_copy_pages", reached)
    cache = fa.Fp4Cache(1, 4, 1, 64, 32, device="cpu")
    a = cache.new()
    batch = cache.batch([a], 3)
    with pytest.raises(ValueError, match="GPU"):
        fa.Fp4Attention(1)(torch.zeros((3, 3 * 64), dtype=torch.bfloat16), batch, 0, torch.zeros((3, 64), dtype=torch.bfloat16))
    b = cache.fork(a)
    with pytest.raises(ValueError, match="GPU"):
        cache.extend(b, 1)
    assert cache.pages_of(a) == cache.pages_of(b) and cache.free_pages() == 3
