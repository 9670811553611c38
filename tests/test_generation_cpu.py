"""Rotation frequencies and the book-keeping of pages (CPU only)."""
import math

import pytest
import torch

from paper_2508_02317_amd import generation as G


def test_frequencies():
    w = G.rope_frequencies(8, base=10000.0)
    assert torch.allclose(w, torch.tensor([1.0, 0.1, 0.01, 0.001], dtype=torch.float64), rtol=1e-14)
    assert torch.equal(G.rope_frequencies(8, scaling="linear", factor=4.0), w / 4)
    b = G.rope_frequencies(8, scaling="base", factor=4.0)
    assert b[0] == 1.0 and abs(b[-1] / w[-1] - 0.25) < 1e-14 and (b[1:-1] < w[1:-1]).all()
    turns = 1000 * w / (2 * math.pi)                                  # 159, 15.9, 1.59, 0.159
    p = G.rope_frequencies(8, scaling="parts", factor=4.0, original=1000, low=1.0, high=32.0)
    assert p[0] == w[0] and torch.isclose(p[3], w[3] / 4, rtol=1e-14)
    for i in (1, 2):
        keep = (turns[i] - 1) / 31
        assert torch.isclose(p[i], w[i] * (keep + (1 - keep) / 4), rtol=1e-14)
    assert G.rope_amplitude(1.0) == 1.0 and abs(G.rope_amplitude(math.e) - 1.1) < 1e-15
    for bad in (dict(rot=7), dict(rot=0), dict(rot=8, factor=0.5), dict(rot=2, scaling="base", factor=2.0), dict(rot=8, scaling="parts"), dict(rot=8, scaling="other"),
                dict(rot=8, scaling="parts", original=100, low=2.0, high=2.0)):
        with pytest.raises(ValueError):
            G.rope_frequencies(**bad)


@pytest.fixture
def cache(monkeypatch):
    monkeypatch.setattr(G.L, "moe_kv_cache", lambda k, v, ks, vs: None)          # no device here
    return G.PagedKVCache(6, 16, 2, 64, device="cpu")


def test_pages_are_handed_out_and_taken_back(cache):
    cache.open("a"); cache.open("b")
    slots, pos, table, lens = cache.grow(["a", "b"], [17, 16])
    assert pos.tolist() == list(range(17)) + list(range(16)) and lens.tolist() == [17, 16]
    assert slots.dtype is torch.int64 and table.dtype is torch.int32 and table.shape == (2, 2)
    assert slots.tolist() == [int(table[0, t // 16]) * 16 + t % 16 for t in range(17)] + [int(table[1, 0]) * 16 + t for t in range(16)]
    assert len(cache.free) == 3 and len(set(cache.pages_of["a"] + cache.pages_of["b"])) == 3
    slots, pos, table, lens = cache.grow(["b"], [1])                            # into a page of its own
    assert pos.tolist() == [16] and slots.tolist() == [int(table[0, 1]) * 16] and len(cache.free) == 2
    before = dict(cache.length), {s: list(p) for s, p in cache.pages_of.items()}, list(cache.free)
    with pytest.raises(MemoryError):
        cache.grow(["a", "b"], [16, 32])                                        # three pages, two free
    assert before == (cache.length, cache.pages_of, cache.free)
    cache.grow(["a"], [0])
    cache.close("a")
    assert len(cache.free) == 4 and "a" not in cache.length
    with pytest.raises(ValueError):
        cache.open("b")
    with pytest.raises(ValueError):
        cache.grow(["b", "b"], [1, 1])
    cache.close("b")
    assert sorted(cache.free) == list(range(6))


def test_counts_that_do_not_fit_change_nothing(cache):
    cache.open("a"); cache.open("b")
    cache.grow(["a", "b"], [5, 20])
    before = dict(cache.length), {s: list(p) for s, p in cache.pages_of.items()}, list(cache.free)
    for counts in ([1], [1, 1, 1], [3, -1]):
        with pytest.raises(ValueError):
            cache.grow(["a", "b"], counts)
        assert before == (cache.length, cache.pages_of, cache.free)
    assert [len(t) for t in cache.grow([], [])] == [0, 0, 0, 0]


def test_rows_that_do_not_fit_leave_the_sequences_as_they_were(cache):
    cache.view = type("View", (), dict(heads=2, dim=64))
    w = torch.zeros((4 + 4) * 64, 32)
    cos = torch.zeros(40, 32)
    attention = G.CachedAttention(cache, 4, w, torch.zeros(32, 4 * 64), cos, cos)
    cache.open("a"); cache.open("b")
    cache.grow(["a", "b"], [40, 3])
    before = dict(cache.length), list(cache.free)
    for call in (lambda: attention.token(torch.zeros(1, 32), ["a"]), lambda: attention.prompt(torch.zeros(39, 32), ["b"], [39]),     # past the table
                 lambda: attention.token(torch.zeros(2, 32), ["b"]), lambda: attention.prompt(torch.zeros(3, 32), ["b"], [4])):          # not as many rows
        with pytest.raises(ValueError):
            call()
        assert before == (cache.length, cache.free)


@pytest.fixture
def attention(cache):
    """Two query heads for each of two key heads of 64 elements, rows of 32, positions up to 40."""
    cache.view = type("View", (), dict(heads=2, dim=64))
    cos = torch.zeros(40, 32)
    return G.CachedAttention(cache, 4, torch.zeros((4 + 4) * 64, 32), torch.zeros(32, 4 * 64), cos, cos)


def state(cache):
    return dict(cache.length), {s: list(p) for s, p in cache.pages_of.items()}, list(cache.free)


@pytest.mark.parametrize("rows", [lambda n: torch.zeros(n, 31), lambda n: torch.zeros(n, 32, dtype=torch.float64), lambda n: torch.zeros(n, 32, dtype=torch.bfloat16),
                                  lambda n: torch.zeros(n, 32, 1), lambda n: torch.zeros(n, 32, device="meta")])
def test_rows_of_another_kind_leave_the_sequences_as_they_were(attention, rows):
    cache = attention.cache
    cache.open("a"); cache.open("b")
    cache.grow(["a", "b"], [15, 3])
    before = state(cache)
    for call in (lambda: attention.token(rows(2), ["a", "b"]), lambda: attention.prompt(rows(22), ["b", "a"], [20, 2])):
        for _ in range(2):
            with pytest.raises((ValueError, TypeError)):
                call()
            assert before == state(cache)


@pytest.mark.parametrize("failing", ["moe_kv_cache_write", "moe_paged_attn_decode", "moe_kv_cache_read", "mm"])
def test_a_step_that_fails_takes_its_growth_back(attention, monkeypatch, failing):
    """Whatever raises after the pages have been handed out: lengths, pages and the order of the free ones are those before the step."""
    cache = attention.cache

    def fail(*_, **__):
        raise MemoryError("no room")

    monkeypatch.setattr(G.L, "moe_kv_cache_write", lambda view, k, v, slots, q, *_, **__: q)
    monkeypatch.setattr(G.L, "moe_paged_attn_decode", lambda q, *_, **__: (q.contiguous(), None))
    monkeypatch.setattr(G.L, "moe_kv_cache_read", lambda *_, rows, **__: (torch.zeros(rows, 2, 64), torch.zeros(rows, 2, 64)))
    cache.open("a"); cache.open("b")
    cache.grow(["a", "b"], [15, 3])
    before = state(cache)
    good = (lambda: attention.token(torch.zeros(2, 32), ["b", "a"]), lambda: attention.prompt(torch.zeros(35, 32), ["b", "a"], [18, 17]))
    with monkeypatch.context() as broken:
        broken.setattr(*((G.torch, "mm") if failing == "mm" else (G.L, failing)), fail)
        for call in good[:1] if failing == "moe_paged_attn_decode" else good[1:] if failing == "moe_kv_cache_read" else good:
            with pytest.raises(MemoryError):
                call()
            assert before == state(cache)
    # the last projection alone
    mm = torch.mm
    with monkeypatch.context() as broken:
        broken.setattr(G.torch, "mm", lambda x, w: fail() if w.shape[1] == 32 else mm(x, w))
        for call in good:
            with pytest.raises(MemoryError):
                call()
            assert before == state(cache)
    assert good[0]().shape == (2, 32) and cache.length == {"a": 16, "b": 4}
    assert good[1]().shape == (35, 32) and cache.length == {"a": 33, "b": 22}


def test_growth_is_taken_back_where_its_tables_cannot_be_made(cache, monkeypatch):
    cache.open("a")
    before = state(cache)
    with monkeypatch.context() as broken:
        broken.setattr(G.torch, "tensor", lambda *_, **__: (_ for _ in ()).throw(RuntimeError("no room")))
        with pytest.raises(RuntimeError):
            cache.grow(["a"], [40])
    assert before == state(cache)


def test_shrink_undoes_grow(cache):
    cache.open("a"); cache.open("b")
    cache.grow(["a", "b"], [17, 1])
    for seqs, counts in ((["a", "b"], [15, 15]), (["b", "a"], [20, 30]), (["a"], [0]), (["b"], [31])):
        before = state(cache)
        cache.grow(seqs, counts)
        cache.shrink(seqs, counts)
        assert before == state(cache)
    cache.shrink(["a"], [17])
    assert cache.length["a"] == 0 and cache.pages_of["a"] == [] and len(cache.free) == 5
    for bad in (["b", "b"], [1, 1]), (["b"], [2]), (["b"], [-1]), (["b"], []):
        before = state(cache)
        with pytest.raises(ValueError):
            cache.shrink(*bad)
        assert before == state(cache)


def test_the_example_keeps_a_bounded_number_of_layers(monkeypatch):
    """A layer's buffers go with its number of rows and are large; prompts come in any number of rows."""
    import os
    import sys
    import weakref
    monkeypatch.syspath_prepend(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import generate
    made = []

    class Layer:
        def __init__(self, rows, *_, **__):
            self.rows = rows
            made.append(weakref.ref(self))

        def forward(self, x):
            assert len(x) == self.rows
            return x

    monkeypatch.setattr(generate, "MoELayer", Layer)
    block = object.__new__(generate.Block)
    block.d = block.experts = block.k = block.f = 1
    block.w_gate = block.w_up = block.w_down = block.w_router = None
    block._layers = {}
    for prompt in range(20, 40):
        for rows in (prompt, 4, 4, 4):
            assert len(block.moe(torch.zeros(rows, 1))) == rows
            assert sum(ref() is not None for ref in made) <= 2
    assert len(made) == 20 + 1                                       # the one of the steps is kept over the prompts
    sys.modules.pop("generate")
