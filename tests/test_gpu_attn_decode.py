"""Attention of one token over a paged cache on the GPU against the fp64 oracle, element by element.

Tolerances, derived.  A score is an fp32 sum of dim exact products, scaled: off by at most (dim + 4) 2^-24 of top = |scale| max_t sum |q k|, and the
exponent 2^x adds x's own rounding, 2^-23 of at most 2 top, and two last places.  p enters the output to 2^-16 (two bf16 numbers, each off by at most 2^-8 of itself; f32: 2^-24); sums of n positive numbers in
chains of n / 16 + 64 are off by that many 2^-24.  All of these multiply sum p |v| / sum p at most twice (numerator and denominator).
The result is rounded once: half a last place."""
import sys

import numpy as np
import pytest

from oracle import attn_oracle as A
from tests.test_gpu_kv_cache import make_cache
from tests.util import to_dev, to_np

pytestmark = pytest.mark.gpu


def say(msg):
    print(msg, flush=True, file=sys.stderr)


def build(kind, lens, Hq, H, D, ps, seed, spare=3, extra_pages=2):
    """A cache in which every place that no sequence owns holds NaN, and every entry of the page table beyond a context a page that does not exist."""
    import torch
    r = np.random.default_rng(seed)
    need = [-(-n // ps) for n in lens]
    pages, max_pages = sum(need) + spare, max(max(need), 1) + extra_pages
    table = np.full((len(lens), max_pages), 1 << 30, dtype=np.int32)
    order = iter(r.permutation(pages))
    cache = make_cache(kind, pages, H, ps, D)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    owned = torch.zeros((pages, ps), dtype=torch.bool)
    for b, n in enumerate(lens):
        for p in range(need[b]):
            table[b, p] = next(order)
            owned[table[b, p], :min(ps, n - p * ps)] = True
    owned = owned.cuda()[:, None, :, None]
    for t, s in ((cache.k, cache.k_scales), (cache.v, cache.v_scales)):
        if kind == "mx8":
            x = torch.randint(0, 256, t.shape, generator=gen, device="cuda").to(torch.uint8)
            x[(x & 0x7F) == 0x7F] = 0x38
            t.copy_(torch.where(owned, x, 0x7F))
            s.copy_(torch.where(owned, torch.randint(116, 122, s.shape, generator=gen, device="cuda").to(torch.uint8), 255))
        else:
            t.copy_(torch.where(owned, torch.randn(t.shape, generator=gen, device="cuda"), float("nan")))
    q = torch.randn((len(lens), Hq, D), generator=gen, device="cuda").to(cache.dtype)
    return cache, q, table, np.array(lens, dtype=np.int32)


def verify(kind, cache, q, table, lens, out, lse, ps, scale, window=0, only=None):
    snap = [None if t is None else to_np(t) for t in (cache.k, cache.v, cache.k_scales, cache.v_scales)]
    got, got_lse, q, D = to_np(out).astype(np.float64), to_np(lse).astype(np.float64), to_np(q), q.shape[2]
    for b in (range(len(lens)) if only is None else only):
        n = int(lens[b])
        lo = max(0, n - window) if window else 0
        k, v = (A.gather(snap[i], snap[2 + i], table[b], ps, lo, n - lo) for i in (0, 1))
        ref, ref_lse, bound, top = A.attend(q[b], k, v, scale)
        if n == 0:
            assert not got[b].any() and np.all(got_lse[b] == -np.inf), b
            continue
        eps = (D + 4) * 2.0 ** -24 * top + 2.0 ** -22 * top + 2.0 ** -22 + (2.0 ** -24 if kind == "f32" else 2.0 ** -16) + ((n - lo) / 16 + 64) * 2.0 ** -24
        tol = 2 * eps[:, None] * bound
        tol = tol + A.half_place(np.abs(ref) + tol, 24 if kind == "f32" else 8)
        bad = ~(np.abs(got[b] - ref) <= tol)
        assert not bad.any(), "sequence %d of %d tokens: %d elements off, worst by %.2g of the bound" % (b, n, bad.sum(), np.nanmax(np.abs(got[b] - ref) / tol))
        bad = ~(np.abs(got_lse[b] - ref_lse) <= 2 * eps + 2.0 ** -22 * np.abs(ref_lse))
        assert not bad.any(), "lse of sequence %d: %s against %s" % (b, got_lse[b][bad][:3], ref_lse[bad][:3])


def run(kind, lens, Hq, H, D, ps, seed=0, window=0, scale=None, **kw):
    from paper_2508_02317_amd import libmoe as L
    say("attend %s lens=%s%s Hq=%d H=%d D=%d page=%d window=%d" % (kind, list(lens)[:12], "..." if len(lens) > 12 else "", Hq, H, D, ps, window))
    cache, q, table, n = build(kind, lens, Hq, H, D, ps, seed)
    out, lse = L.moe_paged_attn_decode(q, cache, to_dev(table), to_dev(n), scale=scale, window=window, lse=True)
    verify(kind, cache, q, table, n, out, lse, ps, D ** -0.5 if scale is None else scale, window, **kw)


EDGES = [0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 0, 511, 513]


@pytest.mark.parametrize("kind", ["f32", "bf16", "mx8"])
@pytest.mark.parametrize("D", [64, 128, 192, 256])
@pytest.mark.parametrize("Hq,H,ps", [(1, 1, 16), (8, 2, 32), (14, 2, 16), (16, 1, 64)])
def test_lengths_around_tiles_and_pages(kind, D, Hq, H, ps):
    run(kind, EDGES, Hq, H, D, ps)


@pytest.mark.parametrize("kind", ["f32", "bf16", "mx8"])
@pytest.mark.parametrize("window", [1, 16, 31, 33, 100, 128, 512, 10000])
def test_windows(kind, window):
    run(kind, EDGES, 8, 4, 128, 16, window=window)


@pytest.mark.parametrize("kind", ["f32", "bf16", "mx8"])
@pytest.mark.parametrize("Hq,H", [(17, 1), (40, 2), (64, 2), (33, 3)])
def test_more_query_heads_than_a_product_has_columns(kind, Hq, H):
    run(kind, [5, 0, 130, 700], Hq, H, 64, 32)


@pytest.mark.parametrize("kind", ["f32", "bf16", "mx8"])
def test_few_long_contexts_are_cut_over_all_workgroups(kind):
    run(kind, [20011, 3], 4, 1, 128, 64)
    run(kind, [9001, 1, 0, 4097], 8, 2, 64, 16, only=[0, 1, 2])


@pytest.mark.parametrize("kind", ["f32", "bf16", "mx8"])
def test_more_sequences_than_a_workgroup_has_threads(kind):
    r = np.random.default_rng(7)
    lens = [int(x) for x in r.integers(0, 60, 700)]
    lens[300:360] = [0] * 60
    run(kind, lens, 2, 2, 64, 16, only=list(range(0, 700, 23)) + [255, 256, 257, 299, 300, 359, 360, 511, 512, 699])


def test_nothing_but_empty_sequences():
    run("bf16", [0, 0, 0], 4, 2, 128, 16)
    from paper_2508_02317_amd import libmoe as L
    cache, q, table, n = build("bf16", [0, 4], 4, 2, 128, 16, 0)
    e = L.moe_paged_attn_decode(q[:0], cache, to_dev(table)[:0].contiguous(), to_dev(n)[:0].contiguous(), lse=True)
    assert e[0].shape == (0, 4, 128)
    out, lse = L.moe_paged_attn_decode(q, cache, to_dev(table)[:, :0].contiguous(), to_dev(n), lse=True)    # no page table at all
    assert not to_np(out).any() and np.all(to_np(lse) == -np.inf)
    out, lse = L.moe_paged_attn_decode(q, cache, to_dev(table), to_dev(np.array([-3, 1 << 30], dtype=np.int32))[[0, 0]].contiguous(), lse=True)
    assert not to_np(out).any()


def test_scores_of_great_range():
    """Scores so far apart that all but one weight vanish, and scales that turn the order round."""
    run("bf16", [300, 77], 8, 2, 128, 16, scale=40.0)
    run("f32", [300, 77], 8, 2, 128, 16, scale=-3.0)
    run("mx8", [300], 8, 2, 128, 16, scale=0.0)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_infinite_and_not_a_number_keys_where_they_count(kind):
    """A key that gives -inf takes part with weight 0; one that gives NaN or +inf makes its head's row NaN and no other."""
    import torch
    from paper_2508_02317_amd import libmoe as L
    cache, q, table, n = build(kind, [400, 90], 4, 2, 64, 16, 3)
    q[...] = q.abs()
    q[..., 0] = 1.0
    cache.k[int(table[0, 0]), 0, 5, 0] = float("-inf")               # the first context, first key head: heads 0 and 1
    cache.k[int(table[1, 2]), 1, 3, 0] = float("nan")                # the second, second key head: heads 2 and 3
    cache.k[int(table[1, 1]), 0, 2, 0] = float("inf")
    out, lse = L.moe_paged_attn_decode(q, cache, to_dev(table), to_dev(n), lse=True)
    assert torch.isfinite(out[0]).all() and torch.isfinite(lse[0]).all()
    assert torch.isnan(out[1]).all()
    verify(kind, cache, q, table, n, out, lse, 16, 64 ** -0.5, only=[]) 
    keep = [t for t in range(400) if t != 5]
    k, v = (A.gather(to_np(x), None, table[0], 16, 0, 400)[keep] for x in (cache.k, cache.v))
    ref, _, bound, _ = A.attend(to_np(q[0]), k, v, 64 ** -0.5)
    assert (np.abs(to_np(out[0])[:2] - ref[:2]) <= 2.0 ** -12 * bound[:2] + A.half_place(np.abs(ref[:2]) + 2.0 ** -12 * bound[:2], 8)).all()


def test_strided_queries_and_another_stream():
    import torch
    from paper_2508_02317_amd import libmoe as L
    cache, q, table, n = build("bf16", [700, 33, 0, 128], 8, 2, 128, 16, 4)
    dev = to_dev(table), to_dev(n)
    ref = L.moe_paged_attn_decode(q, cache, *dev, lse=True)
    whole = torch.full((4, 12, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
    whole[:, 2:10] = q
    got = L.moe_paged_attn_decode(whole[:, 2:10], cache, *dev, lse=True)
    assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = L.moe_paged_attn_decode(q, cache, *dev, lse=True)
    side.synchronize()
    assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])


@pytest.mark.parametrize("kind", ["f32", "bf16", "mx8"])
def test_the_same_call_gives_the_same_bits(kind):
    import torch
    from paper_2508_02317_amd import libmoe as L
    cache, q, table, n = build(kind, [5000, 3, 777, 0, 2500, 64], 8, 2, 128, 32, 5)
    dev = to_dev(table), to_dev(n)
    first = L.moe_paged_attn_decode(q, cache, *dev, lse=True)
    for _ in range(5):
        ws = torch.randint(0, 256, (L.lib.moe_paged_attn_decode_workspace_bytes(6, 8, 2, 128, 32, table.shape[1]),), device="cuda").to(torch.uint8)
        again = L.moe_paged_attn_decode(q, cache, *dev, lse=True, ws=ws)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_a_generation_step_replays_from_a_graph():
    import torch
    from paper_2508_02317_amd import libmoe as L
    cache, q, table, n = build("mx8", [900, 16, 1, 333], 8, 2, 128, 16, 6)
    pages, lens = to_dev(table), to_dev(n)
    r = np.random.default_rng(1)
    k, v = (to_dev(r.standard_normal((4, 2, 128)).astype(np.float32), "bf16") for _ in range(2))
    cos, sin = (to_dev(x.astype(np.float32)) for x in A.rope_table(np.exp(-np.arange(64.0) / 5), 1024))
    pos = to_dev((n - 1).astype(np.int32))
    slots = to_dev(np.array([table[b, (n[b] - 1) // 16] * 16 + (n[b] - 1) % 16 for b in range(4)], dtype=np.int64))
    q_out, out, lse = torch.empty_like(q), torch.empty_like(q), torch.empty((4, 8), device="cuda")
    ws = torch.empty(L.lib.moe_paged_attn_decode_workspace_bytes(4, 8, 2, 128, 16, table.shape[1]), dtype=torch.uint8, device="cuda")

    def step():
        L.moe_kv_cache_write(cache, k, v, slots, q, pos, cos, sin, q_out=q_out)
        L.moe_paged_attn_decode(q_out, cache, pages, lens, out=out, lse=lse, ws=ws)

    step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        step()
    for rep in range(4):
        q.copy_(torch.randn(q.shape, device="cuda"))
        lens.copy_(to_dev(np.maximum(n - rep, 1)))
        step()
        torch.cuda.synchronize()
        ref = [t.clone() for t in (q_out, out, lse, cache.k, cache.k_scales)]
        for t in (q_out, out, lse):
            t.fill_(7.0)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(ref, (q_out, out, lse, cache.k, cache.k_scales))), rep


@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 32, 2 ** 31 - 33, 2 ** 30])
def test_a_window_beyond_every_context_is_none(window):
    import torch
    from paper_2508_02317_amd import libmoe as L
    say("attend, window %d" % window)
    cache, q, table, n = build("bf16", [2500, 3, 0, 700], 8, 2, 128, 16, 8)
    dev = to_dev(table), to_dev(n)
    a, b = (L.moe_paged_attn_decode(q, cache, *dev, window=w, lse=True) for w in (0, window))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("lens", [[400, 90], [20, 3000]])
def test_infinite_and_not_a_number_values_where_they_count(kind, lens):
    """They make their element of their heads' outputs infinite or NaN, and leave every other as it is."""
    import torch
    from paper_2508_02317_amd import libmoe as L
    cache, q, table, n = build(kind, lens, 4, 2, 64, 16, 9)
    dev = to_dev(table), to_dev(n)
    ref, ref_lse = L.moe_paged_attn_decode(q, cache, *dev, lse=True)
    cache.v[int(table[0, 1]), 0, 2, 7] = float("inf")                # first context, token 18: heads 0 and 1
    cache.v[int(table[1, 0]), 1, 3, 60] = float("nan")               # second context, token 3: heads 2 and 3
    out, lse = L.moe_paged_attn_decode(q, cache, *dev, lse=True)
    hit = torch.zeros_like(out, dtype=torch.bool)
    hit[0, :2, 7] = hit[1, 2:, 60] = True
    assert torch.equal(lse, ref_lse) and not torch.isfinite(out[hit]).any() and torch.equal(out[~hit], ref[~hit])


def run_on_a_used_workspace(kind, lens, Hq, H, D, ps, window=0, only=None):
    import torch
    from paper_2508_02317_amd import libmoe as L
    say("attend %s %d sequences of up to %d Hq=%d H=%d D=%d page=%d window=%d, workspace of random bytes" % (kind, len(lens), max(lens), Hq, H, D, ps, window))
    cache, q, table, n = build(kind, lens, Hq, H, D, ps, 11)
    ws = torch.randint(0, 256, (L.lib.moe_paged_attn_decode_workspace_bytes(len(lens), Hq, H, D, ps, table.shape[1]),), device="cuda").to(torch.uint8)
    out, lse = L.moe_paged_attn_decode(q, cache, to_dev(table), to_dev(n), window=window, lse=True, ws=ws)
    verify(kind, cache, q, table, n, out, lse, ps, D ** -0.5, window, only)


@pytest.mark.parametrize("kind", ["f32", "bf16", "mx8"])
@pytest.mark.parametrize("window", [1000, 1017])
@pytest.mark.parametrize("Hq,H,D", [(8, 2, 128), (34, 2, 64), (4, 1, 256)])
def test_windows_that_are_cut_into_pieces(kind, window, Hq, H, D):
    """Windows of 32 stretches and more, which begin far behind the context's first tokens, on and off the multiples of a stretch and a page."""
    run_on_a_used_workspace(kind, [5000, 1700, 0, 1001, 3], Hq, H, D, 16 if D == 64 else 32, window)


@pytest.mark.parametrize("kind", ["f32", "bf16", "mx8"])
@pytest.mark.parametrize("window", [0, 1003])
def test_more_than_256_sequences_of_which_some_are_cut(kind, window):
    r = np.random.default_rng(12)
    lens = [int(x) for x in r.integers(0, 40, 300)]
    for b, n in ((0, 2100), (129, 1500), (251, 3000), (255, 0), (259, 1999), (299, 1501)):
        lens[b] = n
    lens[230:250], lens[254:259] = [0] * 20, [0] * 5
    run_on_a_used_workspace(kind, lens, 4, 2, 64, 16, window, only=[0, 1, 128, 129, 130, 229, 230, 249, 250, 251, 252, 253, 254, 255, 256, 257, 258, 259, 260, 298, 299])


@pytest.mark.parametrize("kind", ["f32", "bf16", "mx8"])
@pytest.mark.parametrize("longest", [600, 1000, 1100])
def test_many_units_around_the_length_from_which_contexts_are_cut(kind, longest):
    """256 units: 32 stretches (1024 tokens, half in fp32 heads of 128) are one piece each, more are cut."""
    r = np.random.default_rng(13)
    lens = [int(x) for x in r.integers(1, longest, 128)]
    lens[5], lens[60], lens[127] = longest, 0, longest - 1
    run_on_a_used_workspace(kind, lens, 4, 2, 128, 16, only=[0, 5, 6, 59, 60, 61, 126, 127])


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("lens", [[400, 90], [3000, 70]])
@pytest.mark.parametrize("bad", ["nan", "inf"])
def test_a_poisoned_key_leaves_the_other_heads_their_bits(kind, lens, bad):
    import torch
    from paper_2508_02317_amd import libmoe as L
    cache, q, table, n = build(kind, lens, 4, 2, 64, 16, 14)
    q[..., 0] = 1.0
    dev = to_dev(table), to_dev(n)
    ref, ref_lse = L.moe_paged_attn_decode(q, cache, *dev, lse=True)
    cache.k[int(table[0, 1]), 0, 2, 0] = float(bad)                  # the first context's token 18: heads 0 and 1
    cache.k[int(table[1, 4]), 1, 3, 0] = float(bad)                  # the second's token 67: heads 2 and 3
    out, lse = L.moe_paged_attn_decode(q, cache, *dev, lse=True)
    hit = torch.zeros((2, 4), dtype=torch.bool, device="cuda")
    hit[0, :2] = hit[1, 2:] = True
    assert torch.isnan(out[hit]).all() and not torch.isfinite(lse[hit]).any()
    assert torch.equal(out[~hit], ref[~hit]) and torch.equal(lse[~hit], ref_lse[~hit])


@pytest.mark.parametrize("k_code,v_code,q_power", [(0, 127, 120), (1, 127, 120), (254, 127, -120), (127, 240, 0)])
def test_scales_at_the_ends_of_their_range(k_code, v_code, q_power):
    """Keys' scales from 2^-127 to 2^127, with queries and a scale that bring the scores back; large ones of values.  Elements from 2 on where scales are the
    smallest (nothing below bf16's normal numbers), up to 1 where they are the largest (no sum beyond fp32's range)."""
    import torch
    from paper_2508_02317_amd import libmoe as L
    cache, q, table, n = build("mx8", [91, 700], 8, 2, 128, 16, 15)
    for t, s, code in ((cache.k, cache.k_scales, k_code), (cache.v, cache.v_scales, v_code)):
        sign, size = t & 0x80, t & 0x7F
        size = torch.where(size == 0x7F, size, size.clamp(min=0x40) if code < 8 else size.clamp(max=0x38) if code > 200 else size)     # 0x7F: places of nobody
        t.copy_(sign | size)
        s.copy_(torch.where(s == 255, s, code))
    q = (q.double() * 2.0 ** q_power).bfloat16()
    scale = float(np.float32(0.01 * 2.0 ** (127 - k_code - q_power)))
    out, lse = L.moe_paged_attn_decode(q, cache, to_dev(table), to_dev(n), scale=scale, lse=True)
    verify("mx8", cache, q, table, n, out, lse, 16, scale)


@pytest.mark.parametrize("D", [64, 128, 192, 256])
def test_the_value_of_a_single_token_comes_out_as_it_is(D):
    """Every code with every scale, down to bf16's smallest numbers: p is 1, so the output is the value, as the cache's reader has it."""
    import torch
    from paper_2508_02317_amd import libmoe as L
    scales, codes = torch.arange(255, device="cuda").to(torch.uint8), torch.arange(256, device="cuda").to(torch.uint8)
    codes[(codes & 0x7F) == 0x7F] = 0x5A                             # but NaN
    for part in codes.split(D) if 256 % D == 0 else (codes[:D], codes[-D:]):
        cache = make_cache("mx8", 255, 1, 16, D)
        cache.v[:, 0, 0] = part
        cache.v_scales[:, 0, 0] = scales[:, None]
        table, lens = torch.arange(255, dtype=torch.int32, device="cuda")[:, None].contiguous(), torch.ones(255, dtype=torch.int32, device="cuda")
        out, _ = L.moe_paged_attn_decode(torch.ones((255, 3, D), dtype=torch.bfloat16, device="cuda"), cache, table, lens)
        _, v = L.moe_kv_cache_read(cache, table, torch.arange(256, dtype=torch.int32, device="cuda"), rows=255)
        ref = A.F.e4m3_decode(to_np(part)) * np.exp2(np.arange(255.0) - 127)[:, None]
        normal = (np.abs(ref) >= 2.0 ** -126) & (np.abs(ref) < 2.0 ** 128)
        assert np.array_equal(to_np(v)[:, 0][normal], ref[normal])
        there = torch.isfinite(v).expand_as(out)
        assert torch.equal(out[there], v.expand_as(out)[there]) and not torch.isfinite(out[~there]).any()
