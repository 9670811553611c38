"""Positions of several axes in generation: the axis of every pair, and the book-keeping of positions beside that of pages (CPU only)."""
import pytest
import torch

from paper_2508_02317_amd import generation as G
from tests.test_generation_cpu import cache, state  # noqa: F401


def test_the_axis_of_every_pair():
    assert G.rope_axes((2, 3, 1)) == bytes([0, 0, 1, 1, 1, 2]) and G.rope_axes((2, 3, 1), cycled=True) == bytes([0, 1, 2, 0, 1, 1])
    assert G.rope_axes((4,)) == bytes(4) and G.rope_axes((0, 2)) == bytes([1, 1]) and len(G.rope_axes((16, 24, 24), True)) == 64
    for bad in ((), (1, 1, 1, 1, 1), (2, -1)):
        with pytest.raises(ValueError):
            G.rope_axes(bad)


@pytest.fixture
def on_axes(cache, monkeypatch):
    """Attention with three axes over the cache, the device's calls replaced; `seen` has the positions of every store."""
    seen = []

    def store(view, k, v, slots, q, positions, cos, sin, axes, interleaved, q_out):
        seen.append(positions.tolist())
        return q

    cache.view = type("View", (), dict(heads=2, dim=64))()
    monkeypatch.setattr(G.L, "moe_kv_cache_write_axes", store)
    monkeypatch.setattr(G.L, "moe_paged_attn_decode", lambda q, *_, **__: (q.contiguous(), None))
    monkeypatch.setattr(G.L, "moe_kv_cache_read", lambda *_, rows, **__: (torch.zeros(rows, 2, 64), torch.zeros(rows, 2, 64)))
    a = G.CachedAttention(cache, 2, torch.zeros(6 * 64, 32), torch.zeros(32, 2 * 64), torch.zeros(40, 32), torch.zeros(40, 32), axes=G.rope_axes((8, 12, 12)))
    a.seen = seen
    return a


def test_positions_go_on_behind_the_largest(on_axes):
    a, cache = on_axes, on_axes.cache
    cache.open("a"); cache.open("b")
    a.prompt(torch.zeros(5, 32), ["a", "b"], [3, 2])
    assert a.seen.pop() == [[0, 1, 2, 0, 1]] * 3 and cache.ahead == {"a": 0, "b": 0}
    picture = torch.tensor([[3, 3, 3, 3, 2], [3, 3, 4, 4, 2], [3, 4, 3, 4, 2]])
    a.prompt(torch.zeros(5, 32), ["a", "b"], [4, 1], picture)
    assert a.seen.pop() == picture.tolist() and cache.length == {"a": 7, "b": 3} and cache.ahead == {"a": -2, "b": 0}
    a.token(torch.zeros(2, 32), ["b", "a"])
    assert a.seen.pop() == [[3, 5]] * 3 and cache.ahead == {"a": -2, "b": 0}
    a.prompt(torch.zeros(1, 32), ["a"], [1], torch.tensor([[20], [9], [9]]))       # a gap
    assert cache.ahead["a"] == 21 - 9
    a.prompt(torch.zeros(2, 32), ["a", "b"], [0, 2])
    assert a.seen.pop() == [[4, 5]] * 3 and cache.ahead["a"] == 12
    cache.close("a")
    assert cache.ahead == {"b": 0}
    cache.open("a")
    a.token(torch.zeros(1, 32), ["a"])
    assert a.seen.pop() == [[0]] * 3


def test_positions_that_do_not_fit_change_nothing(on_axes, monkeypatch):
    a, cache = on_axes, on_axes.cache
    cache.open("a")
    a.prompt(torch.zeros(3, 32), ["a"], [3], torch.tensor([[0, 0, 0], [0, 0, 5], [0, 1, 0]]))
    before = state(cache), dict(cache.ahead)
    three = lambda v: torch.tensor(v).expand(3, -1)
    for seqs, counts in ((['a', 'a'], [1, 1]), (['a'], [-1]), (['a'], []), (['a'], [1, 1])):
        with pytest.raises(ValueError):
            a.prompt(torch.zeros(sum(counts) if sum(counts) > 0 else 0, 32), seqs, counts)
        assert before == (state(cache), cache.ahead)
    for bad in ([[6, 7]] * 3, three([6, 40]), three([-1, 0]), three([6]), torch.zeros(2, 2, dtype=torch.int32), three([6.0, 7.0])):
        with pytest.raises(ValueError):
            a.prompt(torch.zeros(2, 32), ["a"], [2], bad)
        assert before == (state(cache), cache.ahead)
    with pytest.raises(ValueError):                                                 # the text would pass the table's end
        a.prompt(torch.zeros(35, 32), ["a"], [35])
    with monkeypatch.context() as broken:
        broken.setattr(G.torch, "mm", lambda *_: (_ for _ in ()).throw(MemoryError("no room")))
        with pytest.raises(MemoryError):
            a.prompt(torch.zeros(2, 32), ["a"], [2], three([6, 39]))
    assert before == (state(cache), cache.ahead)
    plain = G.CachedAttention(cache, 2, torch.zeros(6 * 64, 32), torch.zeros(32, 2 * 64), torch.zeros(40, 32), torch.zeros(40, 32))
    with pytest.raises(ValueError):
        plain.prompt(torch.zeros(1, 32), ["a"], [1], torch.zeros(3, 1, dtype=torch.int32))
    with pytest.raises(ValueError):
        G.CachedAttention(cache, 2, torch.zeros(6 * 64, 32), torch.zeros(32, 2 * 64), torch.zeros(40, 32), torch.zeros(40, 32), axes=bytes(31))


def test_tokens_taken_back_give_their_positions_back(on_axes):
    """What shrink leaves goes on as if the tokens taken back had never been there: in the text behind a picture, in the picture and before it."""
    a, cache = on_axes, on_axes.cache
    cache.open("a"); cache.open("b")
    rows = lambda n: torch.zeros(n, 32)
    picture = torch.tensor([[4, 4, 4, 4], [4, 4, 5, 5], [4, 5, 4, 6]])
    step = [lambda: a.prompt(rows(4), ["a"], [4]), lambda: a.prompt(rows(4), ["a"], [4], picture), lambda: a.token(rows(1), ["a"]),
            lambda: a.prompt(rows(2), ["a"], [2], torch.tensor([[20, 3]] * 3)), lambda: a.token(rows(1), ["a"])]
    for f in step:
        f()
    follows = [0, 1, 2, 3, 4, 5, 6, 6, 7, 8, 21, 21, 22]                            # position behind the first n tokens
    a.seen.clear()
    for length in (12, 11, 10, 9, 8, 7, 6, 5, 4, 2, 0):
        cache.shrink(["a"], [cache.length["a"] - length])
        a.prompt(rows(3), ["b", "a"], [1, 2])                                       # text goes on, and is taken back
        assert a.seen.pop()[0][1:] == [follows[length], follows[length] + 1]
        cache.shrink(["a", "b"], [2, 1])
        assert cache.length == {"a": length, "b": 0} and cache.ahead == {"a": follows[length] - length, "b": 0}
    assert cache.placed == {"a": [], "b": []}
    for f in step:
        f()
    cache.shrink(["a"], [9])                                                        # over the second picture and all but none of the first
    assert cache.ahead["a"] == 0 and cache.placed["a"] == []
    with pytest.raises(ValueError):
        cache.shrink(["a"], [5])
    cache.close("a")
    assert cache.placed == {"b": []} and cache.ahead == {"b": 0}


@pytest.mark.parametrize("patches", [
    [(0, i // 8, i % 8) for i in range(24)],                                        # in raster order
    [(0, i // 8, i % 8) for i in range(19)],                                        # the same, ending inside a row
    [(0, i % 3, i // 3) for i in range(24)],                                        # column by column
    [(i // 4, 0, 9 - i % 4) for i in range(12)],                                    # frames, each from its last column on
    [(0, 0, i) for i in (11, 3, 7, 0, 2)]])
def test_what_follows_a_picture_is_the_same_however_it_is_cut(on_axes, patches):
    """Behind the first n tokens of a sequence text goes on one behind the largest position that they have, in whichever chunks they came."""
    a, cache = on_axes, on_axes.cache
    rows = lambda n: torch.zeros(n, 32)
    picture, n = torch.tensor(patches).t().contiguous() + 2, len(patches)
    follows = [0, 1, 2] + (picture.amax(0).cummax(0).values + 1).tolist()           # behind two tokens of text and 0, 1, ... patches
    for cut in range(n + 1):
        for length in range(n + 2, -1, -1):
            cache.open("a")
            a.prompt(rows(2), ["a"], [2])
            for part in (picture[:, :cut], picture[:, cut:]):
                a.prompt(rows(part.shape[1]), ["a"], [part.shape[1]], part)
            assert cache.length["a"] + cache.ahead["a"] == follows[-1], cut
            cache.shrink(["a"], [n + 2 - length])
            a.seen.clear()
            a.token(rows(1), ["a"])
            assert a.seen == [[[follows[length]]] * 3], (cut, length)
            cache.close("a")
