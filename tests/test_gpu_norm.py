"""The norm on the GPU against the fp64 oracle, element by element.

Tolerances, derived, with u = 2^-24.  A sum over a row of D <= 16384 elements is a chain of at most 16 or 32 in a lane, 6 steps over a wave and up to 16 over waves,
so at most 54 additions deep, each term with one rounding more: 64 u of the sum of magnitudes covers it.
  forward: mean 64 u mean|h|.  The variance: 64 u from its sum, 2 u a term from the difference and the square, and the square of the mean's error, which is below u
    of mean(h^2) (64 u)^2 -- nothing; rstd takes half of it and 3 roundings: 36 u.  y = (h - m) r w + b: the mean's error, and 36 + 4 u of |(h - m) r w|, and u of |y|.
  backward (mean and rstd are inputs): xh 2 u, g u; mean(g) 65 u of mean|g|, mean(g xh) 69 u of mean|g xh|; the outer sum 3 roundings of its parts.
  sums over rows: at most rows / 256 + 4 terms in a lane (256 workgroups, 4 rows at once), 6 + 16 + 16 + 16 deep beyond, 3 u a term: (64 + rows / 256) u of the
    magnitudes' sum.
In bf16, half a last place of the result more (2^-9 of its binade), also where h is rounded."""
import sys

import numpy as np
import pytest

from oracle import attn_oracle as A
from oracle import train_oracle as O
from tests.util import to_dev, to_np

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
SHAPES = [(1, 1, 8), (3, 1, 64), (5, 1, 200), (17, 1, 1000), (33, 1, 2048), (7, 1, 2056), (4, 1, 4096), (3, 1, 8192), (2, 1, 16384), (2, 1, 16376), (9, 4, 128), (6, 3, 64),
          (11, 28, 192), (5, 2, 256), (700, 7, 16), (1031, 1, 512)]


def say(msg):
    print(msg, flush=True, file=sys.stderr)


def close(got, ref, tol, dtype, what):
    got = to_np(got).astype(np.float64) if hasattr(got, "is_cuda") else np.asarray(got, dtype=np.float64)
    if dtype == "bf16":
        tol = tol + A.half_place(np.abs(ref) + tol, 8)
    bad = ~(np.abs(got - ref) <= tol)
    assert got.shape == ref.shape and not bad.any(), "%s: %d of %d elements off, first %s, %r for %r" % (
        what, bad.sum(), bad.size, np.argwhere(bad)[:3].tolist(), got[bad][:3].tolist(), ref[bad][:3].tolist())


def make(T, H, D, dtype, seed, wdtype="f32"):
    r = np.random.default_rng(seed)
    shape = (T, H, D) if H > 1 else (T, D)
    x = to_dev((r.standard_normal(shape) * np.exp(0.5 * r.standard_normal(D)) + r.standard_normal(shape[:-1] + (1,))).astype(np.float32), dtype)
    other = [to_dev(r.standard_normal(shape).astype(np.float32), dtype) for _ in range(2)]
    w, b = (to_dev(v.astype(np.float32), wdtype) for v in (1 + 0.3 * r.standard_normal(D), r.standard_normal(D)))
    return x, other[0], other[1], w, b


def check_fwd(out, h, w, b, eps, rms, dtype, what):
    y, _, mean, rstd = out
    h, w, b = to_np(h).astype(np.float64), None if w is None else to_np(w), None if b is None else to_np(b)
    ry, rm, rr = O.norm(h, w, b, eps, rms)
    close(rstd, rr, 36 * U * rr, "f32", what + " rstd")
    m_err = np.zeros_like(rm) if rms else 64 * U * np.abs(h).mean(-1)
    if not rms:
        close(mean, rm, m_err, "f32", what + " mean")
    scaled = np.abs(ry if b is None else ry - b)
    close(y, ry, (1.0 if w is None else np.abs(w)) * (rr * m_err)[..., None] + 40 * U * scaled + U * np.abs(ry), dtype, what + " y")


def check_bwd(out, dy, x, mean, rstd, w, add, rms, dtype, wdtype, what):
    dx, dw, db = out
    dy, x, rstd = (to_np(t).astype(np.float64) for t in (dy, x, rstd))
    w, mean, add = (None if t is None else to_np(t).astype(np.float64) for t in (w, mean, add))
    rdx, rdw, rdb = O.norm_bwd(dy, x, mean, rstd, w, add, rms)
    r = rstd[..., None]
    xh = (x if rms else x - mean[..., None]) * r
    g = np.abs(dy if w is None else dy * w)
    mg, mgx = g.mean(-1, keepdims=True), (g * np.abs(xh)).mean(-1, keepdims=True)
    part = U * np.abs(r) * (5 * g + (0 if rms else 70 * mg) + 76 * np.abs(xh) * mgx)
    close(dx, rdx, part + 2 * U * (np.abs(rdx) + (0 if add is None else np.abs(add))), dtype, what + " dx")
    rows = x.size // x.shape[-1]
    for got, ref, size, name in ((dw, rdw, np.abs(dy * xh), "dw"), (db, rdb, np.abs(dy), "db")):
        if got is not None:
            close(got, ref, (64 + rows / 256) * U * size.sum(tuple(range(x.ndim - 1))), wdtype, "%s %s" % (what, name))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("T,H,D", SHAPES)
def test_forward_and_backward(dtype, rms, T, H, D):
    from paper_2508_02317_amd import libmoe as L
    say("norm %s rms=%d T=%d H=%d D=%d" % (dtype, rms, T, H, D))
    for wdtype in {"f32", dtype}:
        x, res, dy, w, b = make(T, H, D, dtype, T + D, wdtype)
        out = L.moe_norm_fwd(x, w, b, 1e-5, rms)
        assert out[1] is None and (out[2] is None) == rms
        check_fwd(out, x, w, b, 1e-5, rms, dtype, "plain")
        with_res = L.moe_norm_fwd(x, w, None, 1e-5, rms, residual=res)
        h = to_np(x).astype(np.float64) + to_np(res)
        close(with_res[1], h, U * np.abs(h), dtype, "h")
        check_fwd(with_res, with_res[1], w, None, 1e-5, rms, dtype, "residual")
        bare = L.moe_norm_fwd(x, None, b, 1e-5, rms)
        check_fwd(bare, x, None, b, 1e-5, rms, dtype, "no weight")
        got = L.moe_norm_bwd(dy, x, out[3], out[2], w, with_bias=True)
        check_bwd(got, dy, x, out[2], out[3], w, None, rms, dtype, wdtype, "plain")
        got = L.moe_norm_bwd(dy, x, out[3], out[2], w, add=res, with_weight=False)
        assert got[1] is None and got[2] is None
        check_bwd(got, dy, x, out[2], out[3], w, res, rms, dtype, wdtype, "add")
        got = L.moe_norm_bwd(dy, x, out[3], out[2], None, with_weight=False, with_bias=True)
        check_bwd(got, dy, x, out[2], out[3], None, None, rms, dtype, "f32", "no weight")


@pytest.mark.parametrize("rms", [False, True])
def test_gradients_are_differences(rms):
    # along random directions, the forward pass in 64 bits: its difference is good to step^2 and 1e-16 / step
    from paper_2508_02317_amd import libmoe as L
    r = np.random.default_rng(9)
    x, dy, v = (r.standard_normal((13, 3, 136)).astype(np.float32) for _ in range(3))
    w, b = (r.standard_normal(136).astype(np.float32) for _ in range(2))
    out = L.moe_norm_fwd(to_dev(x), to_dev(w), to_dev(b), 0.1, rms)
    dx, dw, db = (to_np(t).astype(np.float64) for t in L.moe_norm_bwd(to_dev(dy), to_dev(x), out[3], out[2], to_dev(w), with_bias=True))
    f = lambda x, w, b: (dy.astype(np.float64) * O.norm(x, w, b, 0.1, rms)[0]).sum()
    s = 1e-4
    for grad, at, way in ((dx, 0, v.astype(np.float64)), (dw, 1, v[0, 0].astype(np.float64)), (db, 2, v[0, 1].astype(np.float64))):
        up, down = [x.astype(np.float64), w.astype(np.float64), b.astype(np.float64)], [x.astype(np.float64), w.astype(np.float64), b.astype(np.float64)]
        up[at] = up[at] + s * way
        down[at] = down[at] - s * way
        num, own = (f(*up) - f(*down)) / (2 * s), (grad * way).sum()
        assert abs(num - own) <= 200 * U * np.abs(grad * way).sum() + 1e-6 * np.abs(grad).sum() * s, (at, num, own)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_views_of_larger_tensors_and_in_place(dtype):
    import torch
    from paper_2508_02317_amd import libmoe as L
    for H, D, rms in ((5, 128, True), (2, 64, False), (1, 1024, False), (1, 4096, True), (3, 520, True)):
        whole = torch.randn((37, H + 2, D), device="cuda").to(torch.float32 if dtype == "f32" else torch.bfloat16)
        before, x = whole.clone(), whole[:, 1:H + 1]
        _, res, dy, w, b = make(37, H, D, dtype, 4)
        res, dy = res.view(37, H, D), dy.view(37, H, D)
        dense = L.moe_norm_fwd(x.contiguous(), w, b, rms=rms, residual=res)
        out = L.moe_norm_fwd(x, w, b, rms=rms, residual=res)
        same = lambda p, q: all(a is None and c is None or torch.equal(a, c) for a, c in zip(p, q))
        assert same(dense, out) and torch.equal(whole, before)
        heads_first = torch.empty((H, 37, D), dtype=x.dtype, device="cuda").transpose(0, 1)     # a transposed output, one row apart from the next head's
        L.moe_norm_fwd(x, w, b, rms=rms, residual=res, out=(heads_first, out[1], out[2], out[3]))
        assert torch.equal(heads_first, dense[0])
        grads = L.moe_norm_bwd(dy, dense[1], dense[3], dense[2], w, add=res, with_bias=True)
        assert same(grads, L.moe_norm_bwd(dy, dense[1], dense[3], dense[2], w, add=res, with_bias=True))        # the same call, the same bits
        for alias in range(3):                                            # dx over dy, x or add
            d, h, a = dy.clone(), dense[1].clone(), res.clone()
            got = L.moe_norm_bwd(d, h, dense[3], dense[2], w, add=a, out=((d, h, a)[alias], torch.empty_like(w), torch.empty_like(b)))
            assert same(grads, got), alias
        p, s = whole[:, 1:H + 1].clone(), res.clone()
        got = L.moe_norm_fwd(p, w, b, rms=rms, residual=s, out=(s, p, dense[2], dense[3]))      # y over the residual, the sum over x
        assert torch.equal(s, dense[0]) and torch.equal(p, dense[1])
        s = res.clone()
        got = L.moe_norm_fwd(x, w, b, rms=rms, residual=s, out=(x, s, dense[2], dense[3]))      # y over x, the sum over the residual
        assert torch.equal(x, dense[0]) and torch.equal(s, dense[1]) and torch.equal(whole[:, 0], before[:, 0]) and torch.equal(whole[:, H + 1], before[:, H + 1])


def test_gradients_that_are_one_row_for_all():
    # what the gradient of a sum is: a tensor without strides, beside an added one that is one row per token
    import torch
    from paper_2508_02317_amd import libmoe as L
    x, res, dy, w, b = make(50, 4, 128, "bf16", 11)
    out = L.moe_norm_fwd(x, w, b)
    one, token = dy[:1, :1].expand(50, 4, 128), res[:, :1].expand(50, 4, 128)
    ref = L.moe_norm_bwd(one.contiguous(), x, out[3], out[2], w, add=token.contiguous(), with_bias=True)
    got = L.moe_norm_bwd(one, x, out[3], out[2], w, add=token, with_bias=True)
    assert all(torch.equal(p, q) for p, q in zip(ref, got))
    assert torch.equal(L.moe_norm_fwd(x, w, b, residual=token)[0], L.moe_norm_fwd(x, w, b, residual=token.contiguous())[0])


def test_more_rows_than_workgroups_take_at_once():
    # long walks: sums over many rows, and rows of one lane
    from paper_2508_02317_amd import libmoe as L
    for T, H, D, dtype in ((20011, 1, 2048, "bf16"), (40003, 5, 64, "bf16"), (150001, 1, 8, "f32"), (3001, 1, 8192, "f32")):
        say("norm T=%d H=%d D=%d" % (T, H, D))
        x, res, dy, w, b = make(T, H, D, dtype, 1)
        out = L.moe_norm_fwd(x, w, b, 1e-5, False)
        check_fwd(out, x, w, b, 1e-5, False, dtype, "%d rows" % (T * H))
        check_bwd(L.moe_norm_bwd(dy, x, out[3], out[2], w, add=res, with_bias=True), dy, x, out[2], out[3], w, res, False, dtype, "f32", "%d rows" % (T * H))


def test_no_rows_and_no_outputs_that_are_not_wanted():
    import torch
    from paper_2508_02317_amd import libmoe as L
    x, _, dy, w, b = make(4, 1, 256, "bf16", 2)
    y, h, m, r = L.moe_norm_fwd(x[:0], w, b)
    assert y.shape == (0, 256) and r.shape == (0,)
    dw, db = torch.full_like(w, 7), torch.full_like(b, 7)
    L.moe_norm_bwd(dy[:0], x[:0], r, m, w, out=(x[:0], dw, db))
    assert not dw.any() and not db.any()
    y, h, m, r = L.moe_norm_fwd(x, w, b, stats=False)
    assert m is None and r is None and torch.equal(y, L.moe_norm_fwd(x, w, b)[0])


def test_a_row_with_nan_or_infinity_spoils_itself_only():
    import torch
    from paper_2508_02317_amd import libmoe as L
    for D in (64, 2048, 8192):
        x, _, dy, w, b = make(40, 1, D, "bf16", 3)
        good = L.moe_norm_fwd(x, w, b)
        gx = L.moe_norm_bwd(dy, x, good[3], good[2], w)[0]
        bad = x.clone()
        bad[7, 5], bad[20, D - 1] = float("nan"), float("inf")
        out = L.moe_norm_fwd(bad, w, b)
        bx = L.moe_norm_bwd(dy, bad, out[3], out[2], w)[0]
        rows = [i for i in range(40) if i not in (7, 20)]
        assert torch.equal(out[0][rows], good[0][rows]) and torch.equal(bx[rows], gx[rows])
        assert out[0][7].isnan().all() and out[0][20].isnan().all() and bx[7].isnan().all() and bx[20].isnan().all()


def test_rows_of_equal_and_of_large_elements():
    import torch
    from paper_2508_02317_amd import libmoe as L
    flat = torch.full((3, 512), 5.0, device="cuda")
    y, _, m, r = L.moe_norm_fwd(flat, eps=1e-6)
    assert not y.any() and (m == 5).all() and torch.allclose(r, torch.tensor(1e3, device="cuda"), rtol=1e-6)
    big = torch.randn((3, 512), device="cuda", dtype=torch.float64) * 1e15 + 1e17      # an offset a hundred times the spread
    y = L.moe_norm_fwd(big.float())[0].double()
    ref = O.norm(to_np(big.float()))[0]
    tol = 64 * U * np.abs(to_np(big.float())).mean(-1, keepdims=True) / to_np(big.float()).std(-1, keepdims=True) + 41 * U * np.abs(ref)
    assert (np.abs(to_np(y) - ref) <= tol).all()


def test_rows_far_apart():
    # strides whose offsets pass 32 bits
    import torch
    from paper_2508_02317_amd import libmoe as L
    D, apart = 256, (1 << 30) + 64
    buf = torch.empty(3 * apart + D, dtype=torch.bfloat16, device="cuda")
    far = buf.as_strided((4, D), (apart, 1))
    x, res, dy, w, b = make(4, 1, D, "bf16", 6)
    far.copy_(x)
    near = L.moe_norm_fwd(x, w, b, residual=res)
    out = L.moe_norm_fwd(far, w, b, residual=res)
    assert torch.equal(out[0], near[0]) and torch.equal(out[1], near[1])
    L.moe_norm_bwd(dy, far, near[3], near[2], w, out=(far, torch.empty_like(w), None))
    assert torch.equal(far, L.moe_norm_bwd(dy, x, near[3], near[2], w)[0])


@pytest.mark.parametrize("compiled", [True, False])
def test_both_ways_of_marshalling_and_what_they_refuse(monkeypatch, compiled):
    import torch
    from paper_2508_02317_amd import libmoe as L
    if compiled and L._marshal is None:
        pytest.skip("_marshal.so is not built here")
    x, res, dy, w, b = make(9, 3, 128, "bf16", 8)
    ref = L.moe_norm_fwd(x, w, b, residual=res)
    back = L.moe_norm_bwd(dy, ref[1], ref[3], ref[2], w, add=res, with_bias=True)
    if not compiled:
        monkeypatch.setattr(L, "_marshal", None)
    assert all(torch.equal(p, q) for p, q in zip(ref, L.moe_norm_fwd(x, w, b, residual=res)))
    assert all(torch.equal(p, q) for p, q in zip(back, L.moe_norm_bwd(dy, ref[1], ref[3], ref[2], w, add=res, with_bias=True)))
    y, h, m, r = ref
    for what, call in (("shape", lambda: L.moe_norm_fwd(x, w, b, residual=res[:8])), ("column", lambda: L.moe_norm_fwd(x, w[:64], b)), ("type", lambda: L.moe_norm_fwd(x, w, b.bfloat16())),
                       ("type", lambda: L.moe_norm_fwd(x, w, b, residual=res.float())), ("contiguous", lambda: L.moe_norm_fwd(x.transpose(1, 2).contiguous().transpose(1, 2))),
                       ("float32", lambda: L.moe_norm_fwd(x.half())), ("elements", lambda: L.moe_norm_bwd(dy, x, r[:8], m, w)), ("float32", lambda: L.moe_norm_bwd(dy, x, r.double(), m, w)),
                       ("shape", lambda: L.moe_norm_bwd(dy[:, :2], x, r, m, w)), ("dim", lambda: L.moe_norm_fwd(x[0, 0])), ("device", lambda: L.moe_norm_fwd(x, w.cpu())),
                       ("type", lambda: L.moe_norm_bwd(dy, x, r, m, w, out=(dy, w.bfloat16(), None)))):
        with pytest.raises((ValueError, TypeError), match=what):
            call()
    with pytest.raises(L.MoEError, match="come together"):
        L.moe_norm_fwd(x, w, b, residual=res, out=(y, None, m, r))
    with pytest.raises(L.MoEError, match="workspace"):
        L.moe_norm_bwd(dy, x, r, m, w, ws=torch.empty(64, dtype=torch.uint8, device="cuda"))
    with pytest.raises(L.MoEError, match="D=100"):
        L.moe_norm_fwd(torch.zeros((2, 100), device="cuda"))
