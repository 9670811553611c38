"""Norm, rotation by several axes and the router's losses together, as a training step and as generation use them: the feed-forward half of a block on its
residual stream against automatic differentiation in 64 bits, a step captured into a graph, and prompts with pictures through attention over the cache.

The bar of whole layers is the repository's: 1e-5 of a tensor's largest element in fp32, 2e-2 in bf16 (tests/util.py)."""
import os
import sys

import numpy as np
import pytest

from oracle import attn_oracle as A
from oracle import train_oracle as O
from tests.util import assert_close, to_dev, to_np

pytestmark = pytest.mark.gpu


def say(msg):
    print(msg, flush=True, file=sys.stderr)


def half_block(T, d, E, k, f, dtype, gather, seed=0, **kw):
    """-> NormedMoE and the tensors it was made of and runs on."""
    import torch
    from paper_2508_02317_amd.layer import MoELayer, NormedMoE
    r = np.random.default_rng(seed)
    mk = lambda *s, scale=1.0: to_dev((scale * r.standard_normal(s)).astype(np.float32), dtype)
    t = dict(wr=mk(E, d, scale=0.2), wg=mk(E, f, d, scale=0.1), wu=mk(E, f, d, scale=0.1), wd=mk(E, d, f, scale=0.1), nw=mk(d, scale=0.2) + 1, nb=mk(d, scale=0.2), x=mk(T, d),
             stream=mk(T, d), dy=mk(T, d, scale=1.0 / T), dh=mk(T, d, scale=1.0 / T))
    layer = MoELayer(T, d, E, k, f, t["x"].dtype, t["wg"], t["wu"], t["wd"], w_router=t["wr"], gather=gather, **kw)
    return t, lambda rms: NormedMoE(layer, t["nw"], t["nb"], eps=1e-5, rms=rms)


@pytest.mark.parametrize("rms", [True, False])
@pytest.mark.parametrize("gather", [True, False])
@pytest.mark.parametrize("padded", [False, True])
def test_half_block_against_automatic_differentiation(rms, gather, padded):
    import torch
    T, d, E, k, f = 53, 64, 12, 3, 32
    t, make = half_block(T, d, E, k, f, "f32", gather, balance=0.3, z=0.05)
    block = make(rms)
    valid = torch.arange(T, device="cuda") % 7 < 5 if padded else None
    y, h = block.forward(t["x"], t["stream"], valid=valid)
    g = block.backward(t["dy"], t["dh"])
    leaf = {n: v.double().cpu().requires_grad_(n not in ("dy", "dh")) for n, v in t.items()}
    hh = leaf["x"] + leaf["stream"]
    c = hh if rms else hh - hh.mean(-1, keepdim=True)
    n = c * (c.square().mean(-1, keepdim=True) + 1e-5).rsqrt() * leaf["nw"] + leaf["nb"]
    z = n @ leaf["wr"].t()
    idx, p = block.moe.topk_idx.cpu().long(), torch.softmax(z, 1)
    w = p.gather(1, idx)
    w = w / w.sum(1, keepdim=True)
    each = torch.einsum("efd,td->tef", leaf["wg"], n)
    act = each * torch.sigmoid(each) * torch.einsum("efd,td->tef", leaf["wu"], n)
    out = torch.einsum("edf,tef->ted", leaf["wd"], act)
    yy = (out.gather(1, idx[..., None].expand(-1, -1, d)) * w[..., None]).sum(1)
    ok = torch.ones(T, dtype=torch.bool) if valid is None else valid.cpu()
    m = int(ok.sum())
    counts = torch.bincount(idx[ok].flatten(), minlength=E)
    balance, zloss = E / (k * m) * (counts * p[ok].sum(0) / m).sum(), torch.logsumexp(z[ok], 1).square().mean()
    ((yy * leaf["dy"]).sum() + (hh * leaf["dh"]).sum() + 0.3 * balance + 0.05 * zloss).backward()
    assert np.array_equal(to_np(block.moe.valid_counts), counts.tolist() + [m])
    check = lambda got, ref, what: assert_close(to_np(got), ref.detach().numpy(), "f32", what)
    check(y, yy, "y"); check(h, hh, "h"); check(block.moe.losses, torch.stack((balance, zloss)), "losses")
    check(g, leaf["x"].grad, "dx")
    for got, name in ((block.dweight, "nw"), (block.dbias, "nb"), (block.moe.dw_router, "wr"), (block.moe.dw_gate, "wg"), (block.moe.dw_up, "wu"), (block.moe.dw_down, "wd")):
        check(got, leaf[name].grad, name)


def test_losses_leave_the_rest_of_the_layer_as_it_is():
    import torch
    out = []
    for kw in (dict(), dict(balance=0.0), dict(balance=0.5, z=0.1)):
        t, make = half_block(300, 256, 16, 4, 128, "bf16", True, **kw)
        block = make(True)
        y, _ = block.forward(t["x"], t["stream"])
        block.backward(t["dy"])
        out.append([x.clone() for x in (y, block.moe.dw_down, block.moe.dlogits)])
    assert all(torch.equal(a, b) for a, b in zip(out[0], out[1])) and all(torch.equal(a, b) for a, b in zip(out[0][:2], out[2][:2])) and not torch.equal(out[0][2], out[2][2])
    with pytest.raises(ValueError, match="valid"):
        t, make = half_block(8, 64, 4, 2, 32, "bf16", True)
        make(True).forward(t["x"], t["stream"], valid=torch.ones(8, dtype=torch.bool, device="cuda"))


def _step(T=1100, seed=4):
    """Calls of one step on buffers of its own -> (run, what it writes)"""
    import torch
    from paper_2508_02317_amd import generation as G
    from paper_2508_02317_amd import libmoe as L
    t, make = half_block(T, 256, 32, 4, 128, "bf16", True, seed=seed, balance=0.01, z=0.001)
    block = make(False)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    qkv = torch.randn((T, 12, 128), generator=gen, device="cuda").bfloat16()
    q, k = qkv[:, :8], qkv[:, 8:10]
    qn, kn = (torch.empty((T, h, 128), dtype=torch.bfloat16, device="cuda") for h in (8, 2))
    r = torch.empty((T, 8), device="cuda")
    dq, dw = torch.empty_like(qn), torch.empty(128, device="cuda")
    w = 1 + 0.1 * torch.randn(128, generator=gen, device="cuda")
    cos, sin = L.moe_rope_table(G.rope_frequencies(128).cuda(), 4096)
    pos = torch.randint(0, 4096, (3, T), generator=gen, device="cuda", dtype=torch.int32)
    pair = G.rope_axes((16, 24, 24))
    ws = torch.empty(L.lib.moe_norm_bwd_workspace_bytes(T, 8, 128), dtype=torch.uint8, device="cuda")

    def run():
        L.moe_norm_fwd(q, w, rms=True, out=(qn, None, None, r))                      # the query norm of a fused projection, then the turn
        L.moe_rope_axes_fwd(qn, k, pos, cos, sin, pair, out=(qn, kn))
        block.forward(t["x"], t["stream"])
        block.backward(t["dy"], t["dh"])
        L.moe_rope_axes_bwd(qn, None, pos, cos, sin, pair, out=(dq, None))
        L.moe_norm_bwd(dq, q, r, None, w, out=(dq, dw, None), ws=ws)

    m = block.moe
    return run, [qn, kn, r, dq, dw, block.dh, block.dweight, block.dbias, m.y, m.losses, m.valid_counts, m.importance, m.lse, m.dlogits, m.dw_router, m.dw_gate]


def test_a_step_replays_from_a_graph():
    import torch
    run, outs = _step()
    other, other_outs = _step(T=700, seed=9)
    eager = []
    for f, o in ((run, outs), (other, other_outs)):
        f()
        torch.cuda.synchronize()
        eager.append([x.clone() for x in o])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs = []
    for f in (run, other):
        with torch.cuda.stream(side):
            f()
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            f()
        graphs.append(g)
    for rep in range(4):
        for o in (outs, other_outs):
            for x in o:
                x.fill_(3)                                 # eager work between replays; also proves that a replay rewrites everything
        torch.cuda.synchronize()
        for g in graphs if rep % 2 else reversed(graphs):
            g.replay()
        if rep == 2:
            run()                                          # an eager step behind the replays, the same results
        torch.cuda.synchronize()
        for e, o in zip(eager, (outs, other_outs)):
            assert all(torch.equal(a, b) for a, b in zip(e, o)), "replay %d differs from the eager step" % rep
        say("  replay %d identical to eager" % rep)


def test_steps_on_two_streams():
    import torch
    steps = [_step(T=900, seed=1), _step(T=1300, seed=2)]
    eager = []
    for f, o in steps:
        f()
        torch.cuda.synchronize()
        eager.append([x.clone() for x in o])
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        for s, (f, _) in zip(streams, steps):
            with torch.cuda.stream(s):
                f()
    torch.cuda.synchronize()
    for e, (_, o) in zip(eager, steps):
        assert all(torch.equal(a, b) for a, b in zip(e, o))


@pytest.mark.parametrize("eight_bit", [False, True])
@pytest.mark.parametrize("sections,cycled", [((16, 24, 24), False), ((24, 20, 20), True)])
def test_prompts_with_pictures_and_steps_after_them(eight_bit, sections, cycled):
    """Attention over the cache with positions of three axes against fp64 evaluation over the cache's own contents; queries are those of the oracle."""
    import torch
    from paper_2508_02317_amd import generation as G
    from paper_2508_02317_amd import libmoe as L
    d, heads, kv, dim = 64, 4, 2, 128
    r = np.random.default_rng(7)
    mk = lambda *s, scale=0.1: to_dev((scale * r.standard_normal(s)).astype(np.float32), "bf16")
    axes = G.rope_axes(sections, cycled)
    cos, sin = L.moe_rope_table(G.rope_frequencies(dim, base=1e4).cuda(), 128)
    cache = G.PagedKVCache(24, 16, kv, dim, eight_bit=eight_bit)
    att = G.CachedAttention(cache, heads, mk((heads + 2 * kv) * dim, d), mk(d, heads * dim), cos, sin, axes=axes)
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import generate
    sys.path.pop(0)
    for s in "abc":
        cache.open(s)
    given = {s: [] for s in "abc"}                           # [3, n] positions of all tokens of a sequence

    def step(x, seqs, counts, positions, y):
        qkv = (x @ att.w_qkv.t()).view(len(x), heads + 2 * kv, dim)
        at = 0
        for s, n in zip(seqs, counts):
            p = np.concatenate(given[s] + [positions[:, at:at + n]], axis=1)
            given[s] = [p]
            q = O.rope_axes(to_np(qkv[at:at + n, :heads]), to_np(cos), to_np(sin), p[:, p.shape[1] - n:], axes, False)
            rows = torch.tensor([0, cache.length[s]], dtype=torch.int32, device="cuda")
            table = torch.tensor([cache.pages_of[s]], dtype=torch.int32, device="cuda")
            kk, vv = (to_np(t).astype(np.float64) for t in L.moe_kv_cache_read(cache.view, table, rows, rows=cache.length[s]))
            new = O.rope_axes(to_np(qkv[at:at + n, heads:heads + kv]), to_np(cos), to_np(sin), p[:, p.shape[1] - n:], axes, False)
            # the cache holds the keys turned by their own positions: 2^-9 of a value in bf16.  In 8 bits half a step is 2^-4 of a value, but a block's scale is
            # the power of two that puts its largest element into [256, 512) and codes end at 448: an element just below 512 loses (512 - 448) / 512 = 2^-3
            step_of = np.abs(new).max() * 2.0 ** -3 if eight_bit else np.abs(new) * 2.0 ** -8 + 1e-6
            assert (np.abs(kk[len(kk) - n:] - new) <= step_of).all()
            for i in range(n):
                end = len(kk) - n + i + 1
                o = np.empty((heads, dim))
                for h in range(heads):
                    sc = kk[:end, h // 2] @ q[i, h] * dim ** -0.5
                    w = np.exp(sc - sc.max())
                    o[h] = w @ vv[:end, h // 2] / w.sum()
                ref = o.ravel() @ to_np(att.w_out).astype(np.float64).T
                assert np.linalg.norm(to_np(y[at + i]) - ref) <= 2e-2 * np.linalg.norm(ref), (s, i)
            at += n

    pic = [to_np(generate.picture_then_text(n, 4, 6)) for n in (40, 10, 25)]
    x = mk(75, d, scale=1.0)
    y = att.prompt(x, list("abc"), [40, 10, 25], torch.from_numpy(np.concatenate(pic, axis=1)))
    step(x, "abc", [40, 10, 25], np.concatenate(pic, axis=1), y)
    nxt = {s: int(p.max()) + 1 for s, p in zip("abc", pic)}
    for seqs in ("cab", "ba"):
        x = mk(len(seqs), d, scale=1.0)
        y = att.token(x, list(seqs))
        step(x, seqs, [1] * len(seqs), np.array([[nxt[s] for s in seqs]] * 3), y)
        for s in seqs:
            nxt[s] += 1
    x = mk(7, d, scale=1.0)                                   # more text, then a picture again
    y = att.prompt(x, ["a", "b"], [4, 3])
    step(x, "ab", [4, 3], np.array([[nxt["a"] + i for i in range(4)] + [nxt["b"] + i for i in range(3)]] * 3), y)
    nxt["a"] += 4
    more = to_np(generate.picture_then_text(9, 3, 3)) + nxt["a"]
    y = att.prompt(mk(9, d, scale=1.0), ["a"], [9], torch.from_numpy(more))
    assert cache.length["a"] + cache.ahead["a"] == nxt["a"] + 3


def test_steps_of_no_sequences_and_sequences_of_no_tokens_on_axes():
    import torch
    from paper_2508_02317_amd import generation as G
    from paper_2508_02317_amd import libmoe as L
    cos, sin = L.moe_rope_table(G.rope_frequencies(64).cuda(), 32)
    cache = G.PagedKVCache(4, 16, 1, 64)
    att = G.CachedAttention(cache, 1, torch.randn((192, 32), device="cuda").bfloat16(), torch.randn((32, 64), device="cuda").bfloat16(), cos, sin, axes=G.rope_axes((8, 12, 12)))
    none = torch.zeros((0, 32), dtype=torch.bfloat16, device="cuda")
    assert att.token(none, []).shape == (0, 32) and att.prompt(none, [], []).shape == (0, 32)
    cache.open("a"); cache.open("b")
    assert att.prompt(none, ["a"], [0], torch.zeros((3, 0), dtype=torch.int32)).shape == (0, 32) and cache.ahead == {"a": 0, "b": 0}
    x = torch.randn((3, 32), device="cuda").bfloat16()
    y = att.prompt(x, ["a", "b"], [0, 3])
    assert y.shape == (3, 32) and y.isfinite().all() and cache.length == {"a": 0, "b": 3}


def test_the_example_runs_with_pictures():
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, os.path.join(root, "examples", "generate.py"), "--seqs", "3", "--prompt", "80", "--tokens", "3", "--pictures"], capture_output=True, text=True,
                       timeout=100)
    assert r.returncode == 0 and "3 sequences" in r.stdout and "nan" not in r.stdout, r.stdout + r.stderr[-2000:]


@pytest.mark.parametrize("renorm", [1, 0])
@pytest.mark.parametrize("gather", [True, False])
def test_losses_of_a_layer_that_is_given_its_logits(renorm, gather):
    """backward() needs no logits: they are those that forward() had."""
    import torch
    from paper_2508_02317_amd.layer import MoELayer
    T, d, E, k, f = 61, 64, 12, 3, 32
    r = np.random.default_rng(2)
    mk = lambda *s, scale=1.0: to_dev((scale * r.standard_normal(s)).astype(np.float32))
    wg, wu, wd, x, dy, logits = mk(E, f, d, scale=0.1), mk(E, f, d, scale=0.1), mk(E, d, f, scale=0.1), mk(T, d), mk(T, d, scale=1.0 / T), mk(T, E)
    valid = torch.arange(T, device="cuda") % 5 < 4
    bare = MoELayer(T, d, E, k, f, torch.float32, wg, wu, wd, renorm=renorm, gather=gather)
    y = bare.forward(x, logits=logits).clone()
    ref = [t.clone() for t in bare.backward(dy, logits=logits)]
    layer = MoELayer(T, d, E, k, f, torch.float32, wg, wu, wd, renorm=renorm, gather=gather, balance=0.3, z=0.05)
    for given in (None, logits.clone()):
        assert torch.equal(layer.forward(x, logits=logits, valid=valid), y)
        got = layer.backward(dy) if given is None else layer.backward(dy, logits=given)
        assert all(torch.equal(a, b) for a, b in zip(got[:4], ref[:4]))
        more = O.balance_bwd(to_np(logits), to_np(layer.topk_idx), 0.3, 0.05, to_np(valid), add=to_np(ref[4]))
        assert_close(to_np(got[4]), more, "f32", "dlogits")


def test_halves_on_one_residual_stream_keep_what_their_backward_passes_read():
    """Two halves in a row: the second adds the first one's y to its stream in a buffer of its own, so the first's gradients are those that it has alone."""
    import torch
    T = 70
    (t, make), (_, other) = half_block(T, 256, 16, 4, 128, "bf16", True, balance=0.1), half_block(T, 256, 16, 4, 128, "bf16", True, seed=5)
    first, second = make(True), other(False)
    y, h = first.forward(t["x"], t["stream"])
    held = h.clone()
    y2, h2 = second.forward(y, h)
    assert torch.equal(h, held) and torch.equal(h2, (y.float() + h.float()).bfloat16())
    g = second.backward(t["dy"], t["dh"]).clone()
    dx = first.backward(g, g).clone()
    t3, make3 = half_block(T, 256, 16, 4, 128, "bf16", True, balance=0.1)
    third = make3(True)
    third.forward(t3["x"], t3["stream"])
    assert torch.equal(third.backward(g, g), dx)
    for name in ("dweight", "dbias"):
        assert torch.equal(getattr(third, name), getattr(first, name))
    assert torch.equal(third.moe.dw_down, first.moe.dw_down) and torch.equal(third.moe.dw_router, first.moe.dw_router)
