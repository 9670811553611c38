"""A block that generates through the cache against the same block evaluated anew for every token in 64 bits, and the two ways into the library."""
import os
import sys

import numpy as np
import pytest

from oracle import attn_oracle as A
from oracle import moe_oracle as O
from tests.util import to_np

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def block_of(eight_bit, **kw):
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import generate
    finally:
        sys.path.pop(0)
    return generate, generate.Block(256, 8, 2, 64, 8, 2, 128, pages=40, page_size=16, n_pos=256, eight_bit=eight_bit, seed=3, **kw)


def norm(x):
    return x / np.sqrt((x * x).mean(-1, keepdims=True) + 1e-6)


def evaluated(block, rows):
    """The last row's output of one sequence whose inputs are rows [n, d], everything in float64 and no cache."""
    w = lambda t: to_np(t).astype(np.float64)
    h = norm(rows)
    qkv = (h @ w(block.w_qkv).T).reshape(len(rows), -1, 64)
    cos, sin = w(block.cos)[:len(rows)], w(block.sin)[:len(rows)]
    q, k, v = A.rope(qkv[:, :8], cos, sin, False), A.rope(qkv[:, 8:10], cos, sin, False), qkv[:, 10:]
    y, _, _, _ = A.attend(q[-1], k, v, 64 ** -0.5)
    x = rows[-1] + y.reshape(-1) @ w(block.w_out).T
    h = norm(x)[None]
    fwd = O.moe_layer_fwd(h, h @ w(block.w_router).T, w(block.w_gate), w(block.w_up), w(block.w_down), 2, 1)
    return x + fwd["Y"][0]


@pytest.mark.parametrize("eight_bit", [False, True])
def test_generation_against_evaluation_from_scratch(eight_bit):
    import torch
    generate, block = block_of(eight_bit, base=1e4)
    gen = torch.Generator(device="cuda").manual_seed(1)
    prompts = [torch.randn((n, 256), generator=gen, device="cuda").bfloat16() for n in (1, 17, 40, 64)]
    rows = generate.generate(block, prompts, 6)
    assert rows.shape == (7, 4, 256) and len(block.cache.free) == 40
    got = to_np(rows).astype(np.float64)
    for s, p in enumerate(prompts):
        history = to_np(p).astype(np.float64)
        for t in range(7):
            ref = evaluated(block, history)
            # weights of std 0.02: each half adds a small part of a row of rms 1, rounded to bf16 twice on the way (2^-9 of it in rms each, and as much again
            # for the roundings inside the halves); 8-bit keys and values are 2^-4 off at most, of an attention output of rms 0.1 at most
            tol = 2.0 ** -7 if not eight_bit else 2.0 ** -6
            err = np.linalg.norm(got[t, s] - ref) / np.linalg.norm(ref)
            assert err <= tol, (s, t, err)
            history = np.concatenate([history, got[t, s][None]])


def test_a_window_and_a_scaled_context():
    """token() continues what prompt() began: the same rows come out whether a sequence goes in as one chunk or token by token."""
    import torch
    for window in (0, 20):
        rows = []
        for whole in (True, False):
            generate, block = block_of(False, base=1e4, scaling="parts", factor=4.0, original=64)
            block.attention.window = window
            x = torch.randn((50, 256), generator=torch.Generator(device="cuda").manual_seed(2), device="cuda").bfloat16()
            block.cache.open(0)
            if whole:
                rows.append(block.attention.prompt(x, [0], [50]))
            else:
                rows.append(torch.cat([block.attention.prompt(x[:30], [0], [30])] + [block.attention.token(x[t:t + 1], [0]) for t in range(30, 50)]))
        a, b = (to_np(r).astype(np.float64) for r in rows)
        # the attention outputs agree to the rounding of one bf16 number, as do the projections of them
        assert np.linalg.norm(a - b) <= 2.0 ** -7 * np.linalg.norm(a), window


def test_both_ways_of_marshalling_give_the_same_bits(monkeypatch):
    import torch
    from paper_2508_02317_amd import libmoe as L
    if L._marshal is None:
        pytest.skip("_marshal.so is not built here")
    outs = []
    for compiled in (True, False):
        if not compiled:
            monkeypatch.setattr(L, "_marshal", None)
        generate, block = block_of(True)
        gen = torch.Generator(device="cuda").manual_seed(4)
        prompts = [torch.randn((n, 256), generator=gen, device="cuda").bfloat16() for n in (5, 33)]
        r = generate.generate(block, prompts, 3)
        q = torch.randn((7, 3, 64), generator=gen, device="cuda")
        pos = torch.arange(7, dtype=torch.int32, device="cuda")
        outs.append([r, block.cache.k, block.cache.v_scales, L.moe_rope_fwd(q, None, pos, block.cos, block.sin)[0], L.moe_rope_bwd(None, q, pos, block.cos, block.sin, True)[1]])
    assert all(torch.equal(a, b) for a, b in zip(*outs))


@pytest.mark.parametrize("compiled", [True, False])
def test_refusals_of_the_binding(compiled, monkeypatch):
    import torch
    from paper_2508_02317_amd import libmoe as L
    if compiled and L._marshal is None:
        pytest.skip("_marshal.so is not built here")
    if not compiled:
        monkeypatch.setattr(L, "_marshal", None)
    mk = lambda *s, t=torch.bfloat16: torch.zeros(s, dtype=t, device="cuda")
    i32, f32 = torch.int32, torch.float32
    q, k, pos, cos = mk(4, 2, 64), mk(4, 1, 64), mk(4, t=i32), mk(8, 32, t=f32)
    rope = L.moe_rope_fwd
    for call, err in ((lambda: rope(q.half(), k, pos, cos, cos), TypeError), (lambda: rope(q, k.float(), pos, cos, cos), TypeError), (lambda: rope(q, k[:3], pos, cos, cos), ValueError),
                      (lambda: rope(q[0], k, pos, cos, cos), ValueError), (lambda: rope(q, k, pos[:3], cos, cos), ValueError), (lambda: rope(q, k, pos.long(), cos, cos), TypeError),
                      (lambda: rope(q, k, pos, cos.double(), cos), TypeError), (lambda: rope(q, k, pos, cos, cos[:, :16]), ValueError), (lambda: rope(q.cpu(), k, pos, cos, cos), ValueError),
                      (lambda: rope(q, k, pos, cos, cos, out=(mk(4, 2, 128), mk(4, 1, 64))), ValueError), (lambda: rope(q.transpose(1, 2), None, pos, cos, cos), ValueError),
                      (lambda: rope(q, k, pos, cos[:, ::2], cos[:, ::2]), ValueError),
                      (lambda: rope(mk(4, 2, 60), None, None, None, None), L.MoEError)):
        with pytest.raises(err):
            call()
    cache = L.moe_kv_cache(mk(3, 1, 16, 64), mk(3, 1, 16, 64))
    slots = mk(4, t=torch.int64)
    write = L.moe_kv_cache_write
    for call, err in ((lambda: write(cache, k, k[:3], slots), ValueError), (lambda: write(cache, k, q, slots), ValueError), (lambda: write(cache, k.float(), k, slots), TypeError),
                      (lambda: write(cache, k, k, slots[:3]), ValueError), (lambda: write(cache, k, k, slots.int()), TypeError), (lambda: write(cache, k, k, slots, q[:3]), ValueError),
                      (lambda: write(cache, k, k, slots, q, pos, cos, cos, q_out=mk(4, 3, 64)), ValueError)):
        with pytest.raises(err):
            call()
    pages, lens, rs = mk(4, 2, t=i32), mk(4, t=i32), mk(5, t=i32)
    read, attend = L.moe_kv_cache_read, L.moe_paged_attn_decode
    for call, err in ((lambda: read(cache, pages, rs), ValueError), (lambda: read(cache, pages, rs[:4], rows=1), ValueError), (lambda: read(cache, pages.long(), rs, rows=1), TypeError),
                      (lambda: read(cache, pages, rs, rows=1, first=lens[:2]), ValueError), (lambda: read(cache, pages, rs, out=(mk(2, 2, 64), mk(2, 2, 64))), ValueError),
                      (lambda: read(cache, pages, rs, out=(mk(2, 1, 64, t=f32), mk(2, 1, 64, t=f32))), TypeError),
                      (lambda: attend(q.float(), cache, pages, lens), TypeError), (lambda: attend(mk(4, 2, 128), cache, pages, lens), ValueError),
                      (lambda: attend(q, cache, pages[:3], lens), ValueError), (lambda: attend(q, cache, pages, lens[:3]), ValueError), (lambda: attend(q, cache, pages, lens.long()), TypeError),
                      (lambda: attend(q, cache, pages, lens, out=mk(4, 2, 32)), ValueError), (lambda: attend(q, cache, pages, lens, lse=mk(4, 3, t=f32)), ValueError),
                      (lambda: attend(q, cache, pages, lens, ws=mk(16, t=torch.uint8)), L.MoEError), (lambda: attend(q, cache, pages, lens, window=-1), L.MoEError)):
        with pytest.raises(err):
            call()
    for bad in ((mk(3, 1, 16, 64), mk(3, 1, 16, 128)), (mk(3, 1, 16, 64), mk(3, 1, 16, 64, t=f32)), (mk(3, 1, 16, 64, t=torch.uint8), mk(3, 1, 16, 64, t=torch.uint8)),
                (mk(3, 16, 1, 64).transpose(1, 2), mk(3, 1, 16, 64)), (mk(3, 1, 16, 64), mk(3, 1, 16, 64), mk(3, 1, 16, 2, t=torch.uint8))):
        with pytest.raises(ValueError):
            L.moe_kv_cache(*bad)


@pytest.mark.parametrize("compiled", [True, False])
def test_one_token_or_one_head_has_no_stride(compiled, monkeypatch):
    """A view's stride over one token or one head is never taken, so it may be anything."""
    import torch
    from paper_2508_02317_amd import libmoe as L
    if compiled and L._marshal is None:
        pytest.skip("_marshal.so is not built here")
    if not compiled:
        monkeypatch.setattr(L, "_marshal", None)
    x = torch.randn((8 * 67 * 3,), device="cuda").bfloat16()
    view = lambda T, H, st, sh: x.as_strided((T, H, 64), (st, sh, 1))
    pos = torch.arange(4, dtype=torch.int32, device="cuda")
    cos, sin = L.moe_rope_table(torch.ones(32, dtype=torch.float64, device="cuda"), 8)
    cache = L.moe_kv_cache(*(torch.zeros((2, 1, 16, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2)))
    table, lens = torch.zeros((1, 1), dtype=torch.int32, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda")
    for T, H, st, sh in ((1, 3, 67, 72), (4, 1, 72, 67), (1, 1, 3, 5)):
        q, k = view(T, H, st, sh), view(T, 1, 72 if T > 1 else 67, 67)
        ref = L.moe_rope_fwd(q.contiguous(), k.contiguous(), pos[:T], cos, sin)
        got = L.moe_rope_fwd(q, k, pos[:T], cos, sin)
        assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])
        q_out = L.moe_kv_cache_write(cache, k, k, pos[:T].long(), q, pos[:T], cos, sin)
        assert torch.equal(q_out, ref[0]) and torch.equal(cache.k[0, 0, :T], ref[1][:, 0]) and torch.equal(cache.v[0, 0, :T], k[:, 0])
        out, _ = L.moe_paged_attn_decode(q[:1], cache, table, lens)
        assert torch.equal(out[0], k[0].expand(H, 64))
    with pytest.raises(OverflowError):
        L.moe_paged_attn_decode(q[:1], cache, table, lens, window=2 ** 32 + 1)


def test_steps_of_no_sequences_and_chunks_of_no_tokens():
    import torch
    generate, block = block_of(True, base=1e4)
    none = torch.empty((0, 256), dtype=torch.bfloat16, device="cuda")
    assert block.attention.token(none, []).shape == (0, 256) and block.attention.prompt(none, [], []).shape == (0, 256)
    block.cache.open(0); block.cache.open(1)
    assert block.attention.prompt(none, [0, 1], [0, 0]).shape == (0, 256)
    x = torch.randn((21, 256), generator=torch.Generator(device="cuda").manual_seed(5), device="cuda").bfloat16()
    y = block.attention.prompt(x, [0, 1], [0, 21])                   # one of them has something to say
    block.cache.open(2)
    assert torch.equal(y, block.attention.prompt(x, [2], [21])) and block.cache.length == {0: 0, 1: 21, 2: 21}


@pytest.mark.parametrize("eight_bit", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("window", [0, 12])
def test_prompts_and_steps_of_sharp_heads_element_by_element(eight_bit, interleaved, window):
    """Both ways through the layer, the attention alone: keys, values and queries are known bit for bit, so every element has the tolerance of one attention."""
    import torch
    from paper_2508_02317_amd.generation import CachedAttention, PagedKVCache
    from tests import attn_step as S
    from tests.util import to_dev
    rows, w, w_out, cos, sin = S.inputs(22)
    attention = CachedAttention(PagedKVCache(40, 16, S.KV_HEADS, S.DIM, eight_bit=eight_bit), S.HEADS, to_dev(w, "bf16"), to_dev(w_out, "bf16"), to_dev(cos), to_dev(sin),
                                interleaved, window)
    seqs = list(range(len(rows)))
    for s in seqs:
        attention.cache.open(s)
    y = to_np(attention.prompt(to_dev(np.concatenate([x[:n] for x, n in zip(rows, S.LENGTHS)]), "bf16"), seqs, list(S.LENGTHS)))
    got = [list(part) for part in np.split(y, np.cumsum(S.LENGTHS)[:-1])]
    for i in range(S.STEPS):
        order = seqs[i % 4:] + seqs[:i % 4]                          # in any order
        y = to_np(attention.token(to_dev(np.stack([rows[s][S.LENGTHS[s] + i] for s in order]), "bf16"), order))
        for s, row in zip(order, y):
            got[s].append(row)
    for x, out in zip(rows, got):
        q, k, v = S.projected(x, w, cos, sin, interleaved, eight_bit)
        for t, row in enumerate(out):
            ref, tol = S.expected(q, k, v, t, window)
            bad = ~(np.abs(row.reshape(S.HEADS, S.DIM).astype(np.float64) - ref) <= tol)
            assert not bad.any(), "token %d of %d: %d elements off, worst by %.3g of the bound" % (t, len(x), bad.sum(), (np.abs(row.reshape(ref.shape) - ref) / tol).max())
