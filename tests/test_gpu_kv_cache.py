"""The paged key/value cache on the GPU: what is written, in full and in 8 bits, and what comes back.  Everything here is compared bit for
bit: the rotation's products and sums are rounded one by one in fp32, which numpy repeats, and quantising is exact up to its one rounding."""
import sys

import numpy as np
import pytest

from oracle import attn_oracle as A
from oracle import moe_fp8 as F
from tests.util import q as rounded
from tests.util import to_dev, to_np

pytestmark = pytest.mark.gpu


def say(msg):
    print(msg, flush=True, file=sys.stderr)


def make_cache(kind, pages, heads, ps, D, fill=None):
    """A view over a cache whose every byte is set beforehand, so that stray writes show."""
    import torch
    from paper_2508_02317_amd import libmoe as L
    dt = {"f32": torch.float32, "bf16": torch.bfloat16, "mx8": torch.uint8}[kind]
    mk = lambda *s, t=dt, f=0x5A: torch.full(s, f, dtype=t, device="cuda")
    k, v = mk(pages, heads, ps, D), mk(pages, heads, ps, D, f=0x3C)
    if kind != "mx8":
        return L.moe_kv_cache(k, v)
    return L.moe_kv_cache(k, v, mk(pages, heads, ps, D // 32, f=100), mk(pages, heads, ps, D // 32, f=101))


def snapshot(cache):
    return [None if t is None else to_np(t).copy() for t in (cache.k, cache.v, cache.k_scales, cache.v_scales)]


def store(want, kind, x, scales, slots, ps):
    """The rows x [T, heads, D] (float32) where the slots say."""
    for t, s in enumerate(slots):
        if s < 0 or s >= want.shape[0] * ps:
            continue
        if kind == "mx8":
            want[s // ps, :, s % ps], scales[s // ps, :, s % ps] = F.mx_quantise(x[t])
        else:
            want[s // ps, :, s % ps] = rounded(x[t], kind)


CASES = [("f32", 1, 2, 1, 64, 64, 16, False), ("f32", 37, 4, 2, 192, 96, 32, True), ("bf16", 1, 1, 1, 128, 128, 16, False), ("bf16", 100, 8, 2, 128, 64, 64, True),
         ("bf16", 53, 5, 5, 256, 256, 16, False), ("mx8", 1, 2, 1, 64, 64, 16, True), ("mx8", 77, 8, 2, 128, 128, 32, False), ("mx8", 40, 3, 3, 192, 192, 16, False),
         ("mx8", 29, 4, 1, 256, 128, 128, True), ("mx8", 300, 16, 4, 128, 32, 16, False)]


@pytest.mark.parametrize("kind,T,Hq,H,D,rot,ps,interleaved", CASES)
def test_write(kind, T, Hq, H, D, rot, ps, interleaved):
    from paper_2508_02317_amd import libmoe as L
    import torch
    say("kv write %s T=%d Hq=%d H=%d D=%d rot=%d page=%d" % (kind, T, Hq, H, D, rot, ps))
    r = np.random.default_rng(T * D + ps)
    dt = "f32" if kind == "f32" else "bf16"
    pages = T // ps + 3
    whole = to_dev((r.standard_normal((T, Hq + 2 * H, D)) * np.exp(r.uniform(-3, 3, (T, 1, 1)))).astype(np.float32), dt)
    whole[0, Hq, :32] = 0                                            # a block of zeros
    q, k, v = whole.split([Hq, H, H], dim=1)                         # strided views
    cos, sin = (x.astype(np.float32) for x in A.rope_table(10000.0 ** (-np.arange(0, rot, 2) / rot), 512))
    pos = r.integers(0, 512, T).astype(np.int32)
    slots = r.permutation(pages * ps)[:T].astype(np.int64)
    if T > 4:
        slots[1], slots[3] = -1, pages * ps + 7                      # not stored
    cache = make_cache(kind, pages, H, ps, D)
    want = snapshot(cache)
    q_out = L.moe_kv_cache_write(cache, k, v, to_dev(slots), q, to_dev(pos), to_dev(cos), to_dev(sin), interleaved)
    turn = lambda x: A.rope(to_np(x), cos[pos], sin[pos], interleaved, dtype=np.float32)
    store(want[0], kind, turn(k), want[2], slots, ps)
    store(want[1], kind, to_np(v), want[3], slots, ps)
    for got, ref, name in zip(snapshot(cache), want, ("k", "v", "k_scales", "v_scales")):
        assert ref is None or np.array_equal(got, ref), name
    assert np.array_equal(to_np(q_out), rounded(turn(q), dt))
    # without queries and without a rotation
    bare = make_cache(kind, pages, H, ps, D)
    want = snapshot(bare)
    assert L.moe_kv_cache_write(bare, k, v, to_dev(slots)) is None
    store(want[0], kind, to_np(k), want[2], slots, ps)
    assert np.array_equal(snapshot(bare)[0], want[0])


def test_write_turns_queries_in_place_and_takes_no_tokens():
    import torch
    from paper_2508_02317_amd import libmoe as L
    r = np.random.default_rng(0)
    cache = make_cache("bf16", 4, 2, 16, 128)
    before = snapshot(cache)
    q, k, v = (to_dev(r.standard_normal((20, h, 128)).astype(np.float32), "bf16") for h in (8, 2, 2))
    cos, sin = (to_dev(x.astype(np.float32)) for x in A.rope_table(np.exp(-np.arange(64.0) / 5), 64))
    pos = torch.arange(20, dtype=torch.int32, device="cuda")
    slots = torch.arange(20, device="cuda")
    assert L.moe_kv_cache_write(cache, k[:0], v[:0], slots[:0], q[:0], pos[:0], cos, sin).shape == (0, 8, 128)
    assert all(np.array_equal(a, b) for a, b in zip(snapshot(cache)[:2], before[:2]))
    ref = L.moe_rope_fwd(q, k, pos, cos, sin)
    assert L.moe_kv_cache_write(cache, k, v, slots, q, pos, cos, sin, q_out=q) is q
    assert torch.equal(q, ref[0])
    assert torch.equal(cache.k[0], ref[1][:16].transpose(0, 1)) and torch.equal(cache.v[1, :, :4], v[16:].transpose(0, 1))


@pytest.mark.parametrize("kind,H,D,ps", [("f32", 2, 64, 16), ("f32", 1, 256, 32), ("bf16", 4, 128, 16), ("bf16", 3, 192, 64), ("mx8", 4, 128, 64), ("mx8", 2, 64, 16),
                                         ("mx8", 1, 192, 32), ("mx8", 8, 256, 16)])
@pytest.mark.parametrize("with_first", [False, True])
def test_read(kind, H, D, ps, with_first):
    import torch
    from paper_2508_02317_amd import libmoe as L
    say("kv read %s H=%d D=%d page=%d first=%d" % (kind, H, D, ps, with_first))
    r = np.random.default_rng(D + ps)
    counts = [0, 1, ps - 1, ps, 0, ps + 1, 3 * ps + 5, 0]
    B, max_pages, pages = len(counts), 6, 41
    cache = make_cache(kind, pages, H, ps, D)
    if kind == "mx8":
        codes = np.delete(np.arange(256), [0x7F, 0xFF]).astype(np.uint8)          # all but NaN
        for t, s in ((cache.k, cache.k_scales), (cache.v, cache.v_scales)):
            t.copy_(to_dev(r.choice(codes, t.shape)))
            s.copy_(to_dev(r.integers(0, 255 - 8, s.shape).astype(np.uint8)))
    else:
        for t in (cache.k, cache.v):
            t.copy_(torch.randn(t.shape, device="cuda"))
    table = np.full((B, max_pages), -7, dtype=np.int32)
    order = iter(r.permutation(pages))
    first = np.array([0, 3, 1, 0, 0, ps, 2, 9] if with_first else [0] * B, dtype=np.int32)
    for b, n in enumerate(counts):
        for p in range(-(-(n + first[b]) // ps)):
            table[b, p] = next(order)
    starts = np.r_[0, np.cumsum(counts)].astype(np.int32)
    rows = int(starts[-1])
    out = tuple(torch.full((rows + 3, H, D), 9.0, dtype=cache.dtype, device="cuda") for _ in range(2))
    L.moe_kv_cache_read(cache, to_dev(table), to_dev(starts), first=to_dev(first) if with_first else None, out=out)
    snap = snapshot(cache)
    for i, got in enumerate(out):
        ref = np.concatenate([A.gather(snap[i], snap[2 + i] if kind == "mx8" else None, table[b], ps, int(first[b]), n) for b, n in enumerate(counts)])
        got = to_np(got).astype(np.float64)
        assert (got[rows:] == 9.0).all()                             # rows that no sequence has
        if kind == "mx8":                                            # exact, but for what falls below bf16's smallest numbers (2^-133)
            with np.errstate(over="ignore"):
                keep = np.abs(ref) < 2.0 ** 127
            assert np.array_equal(got[:rows][keep & (np.abs(ref) >= 2.0 ** -126)], ref[keep & (np.abs(ref) >= 2.0 ** -126)])
            assert (np.abs(got[:rows] - ref)[np.abs(ref) < 2.0 ** -126] <= 2.0 ** -134).all()
        else:
            assert np.array_equal(got[:rows], ref)
    fresh = L.moe_kv_cache_read(cache, to_dev(table), to_dev(starts), rows=rows, first=to_dev(first) if with_first else None)
    assert all(torch.equal(a, b[:rows]) for a, b in zip(fresh, out))


def test_read_of_tokens_that_have_no_page_gives_zeros():
    import torch
    from paper_2508_02317_amd import libmoe as L
    cache = make_cache("bf16", 3, 2, 16, 64)
    table = to_dev(np.array([[1, 99], [-1, 2]], dtype=np.int32))
    k, v = L.moe_kv_cache_read(cache, table, to_dev(np.array([0, 40, 60], dtype=np.int32)), rows=60, first=to_dev(np.array([0, 10], dtype=np.int32)))
    there = np.r_[np.ones(16), np.zeros(24), np.zeros(6), np.ones(14)].astype(bool)      # first page; beyond it 99 and past the table; -1; page 2
    for t in (k, v):
        rows = to_np(t).reshape(60, -1)
        assert (rows[there] != 0).all() and (rows[~there] == 0).all()


def test_write_then_read_of_an_8_bit_cache_keeps_a_sixteenth():
    import torch
    from paper_2508_02317_amd import libmoe as L
    cache = make_cache("mx8", 5, 4, 64, 128)
    k, v = (torch.randn((250, 4, 128), device="cuda").bfloat16() for _ in range(2))
    slots = torch.randperm(320, device="cuda")[:250].sort().values
    L.moe_kv_cache_write(cache, k, v, slots)
    table = torch.arange(5, dtype=torch.int32, device="cuda")[None]
    got = L.moe_kv_cache_read(cache, table, to_dev(np.array([0, 320], dtype=np.int32)), rows=320)
    for x, y in zip((k, v), got):
        x, y = x.float(), y[slots].float()
        top = x.unflatten(-1, (-1, 32)).abs().amax(-1, keepdim=True).expand(-1, -1, -1, 32).flatten(-2)
        # 2^-4 of an element; half a step of the smallest numbers of a block below 2^-14 of its maximum; 448 for what lies above (1/8 at most)
        assert ((x - y).abs() <= torch.maximum(torch.maximum(x.abs() / 16, top * 2.0 ** -18), torch.where(x.abs() > top * 0.85, x.abs() / 8, 0))).all()


def test_cache_beyond_32_bits():
    """Pages that begin more than 2^32 elements into the cache, keys and values interleaved in one tensor."""
    import torch
    from paper_2508_02317_amd import libmoe as L
    H, ps, D = 2, 16, 128
    pages = (1 << 32) // (2 * H * ps * D) + 5
    both = torch.empty((pages, 2, H, ps, D), dtype=torch.uint8, device="cuda")
    sc = torch.empty((pages, 2, H, ps, D // 32), dtype=torch.uint8, device="cuda")
    cache = L.moe_kv_cache(both[:, 0], both[:, 1], sc[:, 0], sc[:, 1])
    k, v = (torch.randn((20, H, D), device="cuda").bfloat16() for _ in range(2))
    at = (pages - 2) * ps - 4
    slots = torch.arange(at, at + 20, device="cuda")
    L.moe_kv_cache_write(cache, k, v, slots)
    small = make_cache("mx8", 3, H, ps, D)
    L.moe_kv_cache_write(small, k, v, slots - (pages - 3) * ps)
    assert torch.equal(both[pages - 3:, 0][0, :, 12:], small.k[0, :, 12:]) and torch.equal(both[pages - 2, 1], small.v[1])
    table = to_dev(np.array([[pages - 3, pages - 2]], dtype=np.int32))
    start = to_dev(np.array([0, 20], dtype=np.int32))
    first = to_dev(np.array([12], dtype=np.int32))
    a = L.moe_kv_cache_read(cache, table, start, rows=20, first=first)
    b = L.moe_kv_cache_read(small, table - (pages - 3), start, rows=20, first=first)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    q = torch.randn((1, 8, D), device="cuda").bfloat16()
    lens = to_dev(np.array([32], dtype=np.int32))
    a = L.moe_paged_attn_decode(q, cache, table, lens, window=20)
    b = L.moe_paged_attn_decode(q, small, table - (pages - 3), lens, window=20)
    assert torch.equal(a[0], b[0])


@pytest.mark.parametrize("D", [64, 128, 192])
def test_a_scale_of_255_is_not_a_number_to_every_reader(D):
    """Its block reads as NaN whatever the codes, in the copy and in the attention alike, and no other element does."""
    import torch
    from paper_2508_02317_amd import libmoe as L
    cache = make_cache("mx8", 3, 2, 16, D)
    cache.k_scales.fill_(127); cache.v_scales.fill_(127)
    cache.k.copy_(torch.arange(cache.k.numel(), device="cuda").remainder(0x7F).to(torch.uint8).view(cache.k.shape))
    table = to_dev(np.array([[2, 0]], dtype=np.int32))
    start, lens = to_dev(np.array([0, 20], dtype=np.int32)), to_dev(np.array([20], dtype=np.int32))
    q = torch.randn((1, 2, D), device="cuda").bfloat16()
    whole, (att, _) = L.moe_kv_cache_read(cache, table, start, rows=20), L.moe_paged_attn_decode(q, cache, table, lens)
    cache.k_scales[0, 1, 2, 1] = 255                                 # token 18, second head, elements 32 .. 63
    cache.v_scales[2, 0, 5, 0] = 255                                 # token 5, first head, elements 0 .. 31
    got, (out, lse) = L.moe_kv_cache_read(cache, table, start, rows=20), L.moe_paged_attn_decode(q, cache, table, lens, lse=True)
    for x, ref, (t, h, at) in zip(got, whole, ((18, 1, 32), (5, 0, 0))):
        hit = torch.zeros_like(x, dtype=torch.bool)
        hit[t, h, at:at + 32] = True
        assert torch.isnan(x[hit]).all() and torch.equal(x[~hit], ref[~hit])
    assert torch.isnan(out[0, 1]).all() and torch.isnan(lse[0, 1]) and torch.isfinite(lse[0, 0])
    assert torch.isnan(out[0, 0, :32]).all() and torch.equal(out[0, 0, 32:], att[0, 0, 32:])


@pytest.mark.parametrize("kind,T,Hq,H,D,rot,ps,interleaved", CASES)
def test_a_store_without_queries_or_a_rotation_leaves_keys_and_values_as_they_are(kind, T, Hq, H, D, rot, ps, interleaved):
    """All four tensors of the cache, everything that was not stored into among them."""
    from paper_2508_02317_amd import libmoe as L
    say("kv write alone %s T=%d H=%d D=%d page=%d" % (kind, T, H, D, ps))
    r = np.random.default_rng(T + D)
    k, v = (to_dev((r.standard_normal((T, H, D)) * np.exp(r.uniform(-3, 3, (T, 1, 1)))).astype(np.float32), "f32" if kind == "f32" else "bf16") for _ in range(2))
    pages = T // ps + 2
    slots = r.permutation(pages * ps)[:T].astype(np.int64)
    cache = make_cache(kind, pages, H, ps, D)
    want = snapshot(cache)
    L.moe_kv_cache_write(cache, k, v, to_dev(slots))
    store(want[0], kind, to_np(k), want[2], slots, ps)
    store(want[1], kind, to_np(v), want[3], slots, ps)
    for got, ref, name in zip(snapshot(cache), want, ("k", "v", "k_scales", "v_scales")):
        assert ref is None or np.array_equal(got, ref), name
