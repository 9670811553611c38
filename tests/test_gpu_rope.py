"""Rotary positions on the GPU against the fp64 oracle, element by element.

Tolerances, derived: an output is one fp32 sum of two fp32 products, each rounded: at most 3 roundings of values no larger than |a c| + |b s|,
so 3 * 2^-24 of that; in bf16 half a last place of the result more: 2^(e - 8) for 2^e <= |y| < 2^(e + 1), the e of the value before the rounding."""
import sys

import numpy as np
import pytest

from oracle import attn_oracle as A
from tests.util import to_dev, to_np

pytestmark = pytest.mark.gpu


def say(msg):
    print(msg, flush=True, file=sys.stderr)


def check(got, ref, mag, dtype, what):
    got = np.asarray(got, dtype=np.float64)
    tol = 3 * 2.0 ** -24 * mag
    if dtype == "bf16":
        tol = tol + A.half_place(np.abs(ref) + tol, 8)
    bad = np.abs(got - ref) > tol
    assert np.isfinite(got).all() and not bad.any(), "%s: %d elements off, first %s" % (what, bad.sum(), np.argwhere(bad)[:3])


def inputs(T, Hq, Hk, D, rot, dtype, seed, n_pos=4096):
    import torch
    r = np.random.default_rng(seed)
    q, k = (to_dev(r.standard_normal((T, h, D)).astype(np.float32), dtype) for h in (Hq, Hk))
    cos, sin = A.rope_table(10000.0 ** (-np.arange(0, rot, 2) / max(rot, 1)), n_pos)
    cos, sin = to_dev(cos.astype(np.float32)), to_dev(sin.astype(np.float32))
    pos = to_dev(r.integers(0, n_pos, T).astype(np.int32))
    return q, k, pos, cos, sin


def of_tokens(table, pos):
    return to_np(table)[to_np(pos)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("T,Hq,Hk,D,rot", [(1, 1, 1, 64, 64), (3, 5, 2, 128, 128), (97, 8, 1, 128, 64), (33, 3, 3, 96, 96), (17, 2, 1, 256, 256), (257, 36, 4, 64, 32),
                                           (5, 1, 1, 16, 16), (9, 4, 2, 200, 48), (4, 2, 2, 512, 512), (19, 7, 1, 192, 96)])
def test_forward_and_backward(dtype, interleaved, T, Hq, Hk, D, rot):
    import torch
    from paper_2508_02317_amd import libmoe as L
    say("rope %s %s T=%d Hq=%d Hk=%d D=%d rot=%d" % (dtype, interleaved, T, Hq, Hk, D, rot))
    q, k, pos, cos, sin = inputs(T, Hq, Hk, D, rot, dtype, T + D)
    c, s = of_tokens(cos, pos), of_tokens(sin, pos)
    for call, back in ((L.moe_rope_fwd, False), (L.moe_rope_bwd, True)):
        out = call(q, k, pos, cos, sin, interleaved)
        for x, y, name in zip((q, k), out, "qk"):
            x = to_np(x)
            check(to_np(y), A.rope(x, c, s, interleaved, back), A.rope_magnitude(x, c, s, interleaved), dtype, "%s back=%d" % (name, back))
    # there and back again: the transpose of the turn is its inverse, and <g, R x> = <R^T g, x>
    if dtype == "f32":
        g = torch.randn_like(q)
        y, _ = L.moe_rope_fwd(q, None, pos, cos, sin, interleaved)
        dx, _ = L.moe_rope_bwd(g, None, pos, cos, sin, interleaved)
        a, b = (g.double() * y.double()).sum().item(), (dx.double() * q.double()).sum().item()
        assert abs(a - b) <= 6 * 2.0 ** -24 * (g.double().abs() * y.double().abs()).sum().item() * 2, (a, b)


def test_parts_that_are_not_turned_keep_their_bits_and_places_in_a_larger_tensor():
    import torch
    from paper_2508_02317_amd import libmoe as L
    T, Hq, Hk, D, rot = 41, 6, 2, 128, 32
    _, _, pos, cos, sin = inputs(T, Hq, Hk, D, rot, "bf16", 5)
    whole = torch.randn((T, Hq + 2 * Hk + 1, D), device="cuda").bfloat16()
    whole[0, 0, 40] = float("nan"); whole[1, 1, 50] = float("inf")
    before = whole.clone()
    q, k = whole[:, :Hq], whole[:, Hq:Hq + Hk]
    ref = L.moe_rope_fwd(q.contiguous(), k.contiguous(), pos, cos, sin)
    out = L.moe_rope_fwd(q, k, pos, cos, sin)                        # strided in, dense out
    bits = lambda t: t.contiguous().view(torch.int16)
    assert all(torch.equal(bits(a), bits(b)) for a, b in zip(ref, out))
    assert torch.equal(bits(out[0][..., rot:]), bits(q[..., rot:]))
    got = L.moe_rope_fwd(q, k, pos, cos, sin, out=(q, k))            # in place
    assert got[0] is q and torch.equal(bits(q), bits(ref[0])) and torch.equal(bits(k), bits(ref[1]))
    assert torch.equal(bits(whole[:, Hq + Hk:]), bits(before[:, Hq + Hk:]))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
def test_in_place_is_the_same(dtype, interleaved):
    import torch
    from paper_2508_02317_amd import libmoe as L
    for D, rot in ((128, 128), (192, 64), (64, 48), (512, 512)):
        q, k, pos, cos, sin = inputs(515, 9, 2, D, rot, dtype, 3)
        ref = L.moe_rope_fwd(q, k, pos, cos, sin, interleaved)
        L.moe_rope_fwd(q, k, pos, cos, sin, interleaved, out=(q, k))
        assert torch.equal(q, ref[0]) and torch.equal(k, ref[1]), (D, rot)


def test_no_tokens_no_heads_no_rotation_and_positions_beyond_the_table():
    import torch
    from paper_2508_02317_amd import libmoe as L
    q, k, pos, cos, sin = inputs(8, 2, 1, 64, 64, "bf16", 1, n_pos=16)
    e = L.moe_rope_fwd(q[:0], k[:0], pos[:0], cos, sin)
    assert e[0].shape == (0, 2, 64) and e[1].shape == (0, 1, 64)
    assert L.moe_rope_fwd(q, None, pos, cos, sin)[1] is None and L.moe_rope_fwd(None, k, pos, cos, sin)[0] is None
    same = L.moe_rope_fwd(q, k, None, None, None)
    assert torch.equal(same[0], q) and torch.equal(same[1], k)
    wild = torch.tensor([-5, -1, 0, 15, 16, 1000, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device="cuda")
    a, b = L.moe_rope_fwd(q, k, wild, cos, sin), L.moe_rope_fwd(q, k, wild.clamp(0, 15), cos, sin)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_more_tokens_than_one_launch_has_rows_of_workgroups():
    # 2^20 workgroups of 4 tokens (512 elements a head) and some more: the last ones walk on
    import torch
    from paper_2508_02317_amd import libmoe as L
    T, D = (1 << 22) + 5, 512
    x = torch.zeros((T, 1, D), dtype=torch.bfloat16, device="cuda")
    x[..., 0] = torch.arange(T, device="cuda").bfloat16()[:, None]
    cos, sin = torch.zeros((1, 8), device="cuda"), torch.ones((1, 8), device="cuda")
    y, _ = L.moe_rope_fwd(x, None, torch.zeros(T, dtype=torch.int32, device="cuda"), cos, sin)
    assert torch.equal(y[:, 0, 8], x[:, 0, 0]) and not y[:, 0, 0].any()


def test_table_of_a_long_context():
    import torch
    from paper_2508_02317_amd import libmoe as L
    freq = 1e6 ** (-np.arange(0, 128, 2) / 128)
    n = 200000
    cos, sin = L.moe_rope_table(torch.from_numpy(freq).cuda(), n, 1.25)
    at = np.r_[0:40, n // 3:n // 3 + 40, n - 40:n]
    a = at[:, None].astype(np.longdouble) * freq.astype(np.longdouble)
    for got, f in ((cos, np.cos), (sin, np.sin)):
        ref = (f(a) * 1.25).astype(np.float64)
        # one rounding to fp32; the angle in fp64 is p 2^-53 off before its reduction
        tol = 2.0 ** -24 * np.abs(ref) + 1.25 * 4 * a.astype(np.float64) * 2.0 ** -53 + 1e-45
        assert (np.abs(to_np(got)[at].astype(np.float64) - ref) <= tol).all()
    assert L.moe_rope_table(torch.from_numpy(freq).cuda(), 0)[0].shape == (0, 64)
