"""Rotary positions with several axes on the GPU: bit for bit the rotation with one axis whose table has been gathered pair by pair beforehand, and against the
fp64 oracle (tolerances as in tests/test_gpu_rope.py); the store into a cache likewise."""
import sys

import numpy as np
import pytest

from oracle import attn_oracle as A
from oracle import train_oracle as O
from tests.test_gpu_rope import check
from tests.util import to_dev, to_np

pytestmark = pytest.mark.gpu


def say(msg):
    print(msg, flush=True, file=sys.stderr)


def pair_axes(half, axes, layout, seed=0):
    if layout == "cycled":
        return bytes(i % axes for i in range(half))
    if layout == "sections":                           # whole eights, so that no lane's pairs differ
        return bytes(min(i // max(8, half // axes // 8 * 8), axes - 1) for i in range(half))
    if layout == "uneven":
        return bytes(min(i // max(1, (half + 2) // axes), axes - 1) for i in range(half))
    return bytes(np.random.default_rng(seed).integers(0, axes, half).astype(np.uint8))


def inputs(T, Hq, Hk, D, rot, axes, dtype, seed, n_pos=4096):
    r = np.random.default_rng(seed)
    q, k, v = (to_dev(r.standard_normal((T, h, D)).astype(np.float32), dtype) for h in (Hq, Hk, Hk))
    cos, sin = A.rope_table(10000.0 ** (-np.arange(0, rot, 2) / rot), n_pos)
    pos = to_dev(r.integers(0, n_pos, (axes, T)).astype(np.int32))
    return q, k, v, pos, to_dev(cos.astype(np.float32)), to_dev(sin.astype(np.float32))


def gathered(cos, sin, pos, pair_axis):
    """The table and positions of the rotation with one axis that does the same."""
    import torch
    c, s = (to_dev(O.axes_table(to_np(t), to_np(pos), pair_axis)) for t in (cos, sin))
    return torch.arange(len(c), dtype=torch.int32, device="cuda"), c, s


def bits(t):
    import torch
    return t.contiguous().view({2: torch.int16, 4: torch.int32, 1: torch.uint8}[t.element_size()])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("layout", ["sections", "uneven", "cycled", "any"])
def test_forward_and_backward(dtype, interleaved, layout):
    import torch
    from paper_2508_02317_amd import libmoe as L
    for T, Hq, Hk, D, rot, axes in ((1, 1, 1, 64, 64, 3), (33, 5, 2, 128, 128, 3), (97, 8, 1, 128, 64, 2), (17, 2, 1, 256, 256, 4), (257, 36, 4, 64, 32, 3), (5, 1, 1, 16, 16, 2),
                                    (9, 4, 2, 200, 48, 4), (4, 2, 2, 512, 512, 3), (19, 7, 1, 192, 96, 1), (40, 3, 3, 96, 96, 3)):
        say("axes %s %s %s T=%d Hq=%d Hk=%d D=%d rot=%d axes=%d" % (dtype, interleaved, layout, T, Hq, Hk, D, rot, axes))
        q, k, _, pos, cos, sin = inputs(T, Hq, Hk, D, rot, axes, dtype, T + D)
        pair = pair_axes(rot // 2, axes, layout)
        one = gathered(cos, sin, pos, pair)
        for call, plain, back in ((L.moe_rope_axes_fwd, L.moe_rope_fwd, False), (L.moe_rope_axes_bwd, L.moe_rope_bwd, True)):
            out, ref = call(q, k, pos, cos, sin, pair, interleaved), plain(q, k, *one, interleaved)
            assert torch.equal(bits(out[0]), bits(ref[0])) and torch.equal(bits(out[1]), bits(ref[1]))
            for x, y, name in zip((q, k), out, "qk"):
                x = to_np(x)
                check(to_np(y), O.rope_axes(x, to_np(cos), to_np(sin), to_np(pos), pair, interleaved, back), A.rope_magnitude(x, to_np(one[1]), to_np(one[2]), interleaved), dtype,
                      "%s back=%d" % (name, back))
        inplace = q.clone()
        assert torch.equal(bits(L.moe_rope_axes_fwd(inplace, None, pos, cos, sin, pair, interleaved, out=(inplace, None))[0]),
                           bits(L.moe_rope_axes_fwd(q, None, pos, cos, sin, pair, interleaved)[0]))


def test_the_gradient_is_the_transpose():
    import torch
    from paper_2508_02317_amd import libmoe as L
    q, _, _, pos, cos, sin = inputs(65, 3, 1, 128, 96, 3, "f32", 2)
    pair, g = pair_axes(48, 3, "uneven"), torch.randn_like(q)
    y, dx = L.moe_rope_axes_fwd(q, None, pos, cos, sin, pair)[0], L.moe_rope_axes_bwd(g, None, pos, cos, sin, pair)[0]
    a, b = (g.double() * y.double()).sum().item(), (dx.double() * q.double()).sum().item()
    assert abs(a - b) <= 2 * 6 * 2.0 ** -24 * (g.double().abs() * y.double().abs()).sum().item(), (a, b)
    # a turn is linear: its difference along any direction is the turn of the direction
    v = torch.randn_like(q)
    d = (L.moe_rope_axes_fwd(q + v, None, pos, cos, sin, pair)[0].double() - L.moe_rope_axes_fwd(q - v, None, pos, cos, sin, pair)[0].double()) / 2
    turned = L.moe_rope_axes_fwd(v, None, pos, cos, sin, pair)[0].double()
    assert (d - turned).abs().max() <= 8 * 3 * 2.0 ** -24 * (q.abs().max() + v.abs().max()).double() * 2


def test_views_and_positions_beyond_the_table():
    import torch
    from paper_2508_02317_amd import libmoe as L
    _, _, _, pos, cos, sin = inputs(23, 1, 1, 128, 128, 3, "bf16", 5, n_pos=64)
    whole = torch.randn((23, 9, 128), device="cuda").bfloat16()
    before, q, k, pair = whole.clone(), whole[:, :6], whole[:, 6:8], pair_axes(64, 3, "sections")
    wild = pos.clone()
    wild[0, 0], wild[1, 1], wild[2, 2], wild[0, 3], wild[1, 4] = -1, 64, 2 ** 31 - 1, -2 ** 31, 1000
    ref = L.moe_rope_axes_fwd(q.contiguous(), k.contiguous(), wild.clamp(0, 63), cos, sin, pair)
    out = L.moe_rope_axes_fwd(q, k, wild, cos, sin, pair, out=(q, k))
    assert torch.equal(out[0], ref[0]) and torch.equal(out[1], ref[1]) and torch.equal(whole[:, 8], before[:, 8])
    empty = L.moe_rope_axes_fwd(q[:0], k[:0], pos[:, :0].contiguous(), cos, sin, pair)
    assert empty[0].shape == (0, 6, 128)


@pytest.mark.parametrize("kind", ["f32", "bf16", "mx8"])
@pytest.mark.parametrize("interleaved", [False, True])
def test_store_into_a_cache(kind, interleaved):
    import torch
    from paper_2508_02317_amd import libmoe as L
    dtype = "f32" if kind == "f32" else "bf16"
    for T, H, Hq, D, rot, axes, layout in ((1, 2, 8, 128, 128, 3, "sections"), (50, 3, 5, 64, 64, 3, "cycled"), (33, 1, 0, 256, 128, 2, "uneven"), (20, 2, 2, 192, 192, 4, "any")):
        say("store %s %s T=%d H=%d D=%d %s" % (kind, interleaved, T, H, D, layout))
        q, k, v, pos, cos, sin = inputs(T, Hq, H, D, rot, axes, dtype, T)
        pair = pair_axes(rot // 2, axes, layout)
        slots = torch.randperm(6 * 16, device="cuda")[:T].contiguous()
        if T > 2:
            slots[1], slots[2] = -1, 6 * 16                              # left out
        got = []
        for axes_call in (True, False):
            mk = lambda n, t: torch.full((6, H, 16, n), 3, dtype=t, device="cuda")
            if kind == "mx8":
                parts = [mk(D, torch.uint8), mk(D, torch.uint8), mk(D // 32, torch.uint8), mk(D // 32, torch.uint8)]
            else:
                parts = [mk(D, q.dtype), mk(D, q.dtype)]
            cache = L.moe_kv_cache(*parts)
            some = q if Hq else None
            if axes_call:
                out = L.moe_kv_cache_write_axes(cache, k, v, slots, some, pos, cos, sin, pair, interleaved)
            else:
                out = L.moe_kv_cache_write(cache, k, v, slots, some, *gathered(cos, sin, pos, pair), interleaved)
            got.append(parts + ([out] if Hq else []))
        assert all(torch.equal(bits(a), bits(b)) for a, b in zip(*got))


@pytest.mark.parametrize("compiled", [True, False])
def test_both_ways_of_marshalling_and_what_they_refuse(monkeypatch, compiled):
    import torch
    from paper_2508_02317_amd import libmoe as L
    if compiled and L._marshal is None:
        pytest.skip("_marshal.so is not built here")
    q, k, v, pos, cos, sin = inputs(9, 4, 2, 64, 64, 3, "bf16", 1)
    pair, slots = pair_axes(32, 3, "any"), torch.arange(9, device="cuda")
    ref = L.moe_rope_axes_fwd(q, k, pos, cos, sin, pair)
    if not compiled:
        monkeypatch.setattr(L, "_marshal", None)
    out = L.moe_rope_axes_fwd(q, k, pos, cos, sin, pair)
    assert torch.equal(out[0], ref[0]) and torch.equal(out[1], ref[1])
    kc, vc = (torch.zeros((2, 2, 16, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    cache = L.moe_kv_cache(kc, vc)
    assert torch.equal(L.moe_kv_cache_write_axes(cache, k, v, slots, q, pos, cos, sin, pair), ref[0]) and torch.equal(kc.transpose(1, 2)[0, :9], ref[1])
    turn = lambda **kw: L.moe_rope_axes_fwd(**dict(dict(q=q, k=k, positions=pos, cos=cos, sin=sin, pair_axis=pair), **kw))
    store = lambda **kw: L.moe_kv_cache_write_axes(**dict(dict(cache=cache, k=k, v=v, slots=slots, q=q, positions=pos, cos=cos, sin=sin, pair_axis=pair), **kw))
    for call in (turn, store):
        for what, bad in (("bytes", dict(pair_axis=list(pair))), ("one entry per pair", dict(pair_axis=pair[:31])), ("must be given", dict(cos=None)), ("axes", dict(positions=pos[0])),
                          ("axes", dict(positions=pos[:, :8].contiguous())), ("contiguous", dict(positions=pos.t().contiguous().t())), ("int32", dict(positions=pos.long())),
                          ("float32", dict(cos=cos.double())), ("device", dict(positions=pos.cpu())), ("cos and sin", dict(sin=sin[:8]))):
            with pytest.raises((ValueError, TypeError), match=what):
                call(**bad)
        for bad in (dict(positions=pos[:2].contiguous()), dict(positions=torch.cat((pos, pos))), dict(pair_axis=b"\3" * 32)):
            with pytest.raises(L.MoEError):
                call(**bad)
    with pytest.raises(ValueError, match="slots"):
        store(slots=slots[:8])
