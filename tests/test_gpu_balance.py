"""The router's losses on the GPU against the fp64 oracle, element by element; counts exactly.

Tolerances, derived, with u = 2^-24.  A probability exp(z - top) / total: the difference and its product with log2 e are off by u |z - top| each, the power of two by
2 u, the total by its terms' errors (the large ones have a small |z - top|) and a sum of depth at most 16 + 6, the reciprocal and the product by 2 u:
(2 R + 32) u relative, R the largest |z - top| of the row's finite logits.
  lse = top + log(total): that of the total, 3 u of log, u of the sum: (R + 28 + 3 |log total| + |lse|) u.
  importance: all terms are positive: (2 R + 32) u and the depth of the sum: T / 256 + 4 in a lane, 6 + 8 in a workgroup, 64 + 16 in the join.
  losses[0]: the same and 4 u.  losses[1]: 2 |lse| times lse's error, and the depth's.
  dlogits: p = exp(z - lse), from lse's own error, the difference and exp: (R + |lse| + 30 + ...) u, taken as the sum above; share 4 u; mean over E terms of depth 22."""
import sys

import numpy as np
import pytest

from oracle import train_oracle as O
from tests.util import to_dev, to_np

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
SHAPES = [(1, 1, 1), (1, 8, 2), (256, 8, 2), (63, 2, 1), (700, 3, 3), (129, 37, 5), (1000, 128, 8), (65, 128, 8), (2047, 64, 6), (33, 1000, 16), (300, 1024, 8), (77, 1023, 3), (9, 301, 64),
          (512, 260, 4), (5000, 16, 1), (3, 128, 64), (20000, 128, 8)]


def say(msg):
    print(msg, flush=True, file=sys.stderr)


def make(T, E, k, seed, padding=0.0, spread=1.5):
    r = np.random.default_rng(seed)
    z = (spread * r.standard_normal((T, E)) + 0.7 * r.standard_normal(E)).astype(np.float32)
    idx = np.argsort(-z, axis=1, kind="stable")[:, :k].astype(np.int32)
    valid = (r.random(T) >= padding) if padding else None
    return z, idx, valid, (1e-3 * r.standard_normal((T, E)) / T).astype(np.float32)


def check(z, idx, valid, add, a, b, dl=None, z_dev=None):
    import torch
    from paper_2508_02317_amd import libmoe as L
    T, E = z.shape
    zd, vd = to_dev(z) if z_dev is None else z_dev, None if valid is None else to_dev(valid)
    out = L.moe_balance_loss_fwd(zd, to_dev(idx), vd)
    again = L.moe_balance_loss_fwd(zd, to_dev(idx), vd)
    assert all(torch.equal(p, q) for p, q in zip(out, again))
    losses, counts, imp, lse = (to_np(t).astype(np.float64) for t in out)
    r_loss, r_counts, r_imp, r_lse, p = O.balance_fwd(z, idx, valid)
    assert np.array_equal(counts, r_counts)
    ok = np.ones(T, bool) if valid is None else np.asarray(valid).astype(bool)
    n, finite = max(int(r_counts[-1]), 1), np.where(np.isfinite(z) & ok[:, None], z, np.nan)
    with np.errstate(all="ignore"):
        top = np.nan_to_num(np.nanmax(finite, axis=1, initial=-np.inf), neginf=0.0)
        R = np.nan_to_num(top - np.nanmin(finite, axis=1, initial=np.inf), neginf=0.0).clip(0)
    known = np.where(np.isfinite(r_lse), r_lse, 0.0)
    lse_tol = U * (R + 28 + 3 * np.abs(known - top) + np.abs(known)) * ok
    assert np.array_equal(np.isinf(lse), np.isinf(r_lse)) and (np.abs(np.where(np.isinf(lse), 0, lse) - known) <= lse_tol).all()
    depth = T / 256 + 98
    p_tol = (2 * R + 32)[:, None] * U * p
    imp_tol = p_tol.sum(0) / n + depth * U * r_imp
    assert (np.abs(imp - r_imp) <= imp_tol).all(), np.abs(imp - r_imp).max()
    share = r_counts[:E] * E / (idx.shape[1] * n)
    assert abs(losses[0] - r_loss[0]) <= (share * imp_tol).sum() + 8 * U * r_loss[0]
    # a mean of squares beyond fp32's range (3.4e38; an lse of 3e38 has the square 9e76) has no other fp32 value than infinity
    assert losses[1] == np.inf if r_loss[1] > np.finfo(np.float32).max else abs(losses[1] - r_loss[1]) <= (2 * np.abs(known) * lse_tol + lse_tol ** 2).sum() / n + (depth + 4) * U * r_loss[1]
    got = L.moe_balance_loss_bwd(zd, out[1], out[3], idx.shape[1], a, b, dlosses=None if dl is None else to_dev(np.float32(dl)), valid=vd, add=None if add is None else to_dev(add))
    sa, sb = (a, b) if dl is None else (a * np.float64(np.float32(dl[0])), b * np.float64(np.float32(dl[1])))
    ref = O.balance_bwd(z, idx, sa, sb, valid, add)
    pb_tol = p * ((2 * R + 34)[:, None] * U + 2 * lse_tol[:, None])
    mean = (p @ share)[:, None]
    tol = (pb_tol * (abs(sa) / n * (share + mean) + abs(sb) * 2 / n * np.abs(known)[:, None]) + p * abs(sa) / n * (6 * U * (share + mean) + 24 * U * mean + (pb_tol @ share)[:, None]) +
           p * abs(sb) * 2 / n * (lse_tol + 6 * U * np.abs(known))[:, None] + 4 * U * np.abs(ref) + (0 if add is None else U * np.abs(add)))
    err = np.abs(to_np(got).astype(np.float64) - ref)
    assert (err <= tol).all(), "dlogits: %d off, %g against %g" % ((err > tol).sum(), err.max(), tol[err > tol][0])
    return out, got


@pytest.mark.parametrize("T,E,k", SHAPES)
def test_losses_and_gradient(T, E, k):
    say("balance T=%d E=%d k=%d" % (T, E, k))
    z, idx, valid, add = make(T, E, k, T + E)
    check(z, idx, None, None, 0.01, 0.001)
    z, idx, valid, add = make(T, E, k, T + E + 1, padding=0.3)
    check(z, idx, valid, add, 0.01, 0.0, dl=(0.5, 3.0))
    check(z, idx, valid.astype(np.uint8) * 200, add, 0.0, 1.0)


def test_gradient_is_the_difference():
    # of the kernel's own losses would drown in their rounding: of the oracle's, along a direction
    from paper_2508_02317_amd import libmoe as L
    z, idx, valid, _ = make(50, 36, 4, 3, padding=0.2)
    out = L.moe_balance_loss_fwd(to_dev(z), to_dev(idx), to_dev(valid))
    g = to_np(L.moe_balance_loss_bwd(to_dev(z), out[1], out[3], 4, 0.7, 0.3, valid=to_dev(valid))).astype(np.float64)
    v, s = np.random.default_rng(4).standard_normal(z.shape), 1e-4
    f = lambda d: O.balance_fwd(z + d * v, idx, valid)[0] @ [0.7, 0.3]
    assert abs((f(s) - f(-s)) / (2 * s) - (g * v).sum()) <= 200 * U * np.abs(g * v).sum() + 1e-6 * s * np.abs(g).sum()


def test_padding_may_hold_anything_and_all_may_be_padding():
    import torch
    from paper_2508_02317_amd import libmoe as L
    for T, E in ((40, 128), (3000, 60), (77, 13)):
        z, idx, valid, add = make(T, E, 3, 8, padding=0.4)
        clean, wild = z.copy(), z.copy()
        wild[~valid] = np.nan
        wild[np.flatnonzero(~valid)[::2]] = np.inf
        wild_idx = idx.copy()
        wild_idx[~valid] = 2 ** 31 - 1
        a, ga = check(clean, idx, valid, add, 0.01, 0.01)
        b = L.moe_balance_loss_fwd(to_dev(wild), to_dev(wild_idx), to_dev(valid))
        gb = L.moe_balance_loss_bwd(to_dev(wild), b[1], b[3], 3, 0.01, 0.01, valid=to_dev(valid), add=to_dev(add))
        assert all(torch.equal(p, q) for p, q in zip(a, b)) and torch.equal(ga, gb) and np.array_equal(to_np(gb)[~valid], add[~valid])
        none = np.zeros(T, bool)
        c = L.moe_balance_loss_fwd(to_dev(wild), to_dev(idx), to_dev(none))
        assert not any(t.any() for t in c)
        assert not L.moe_balance_loss_bwd(to_dev(wild), c[1], c[3], 3, 1.0, 1.0, valid=to_dev(none)).any()


def test_logits_of_minus_infinity_and_far_apart():
    for E in (8, 13, 512):
        z, idx, _, add = make(30, E, 2, E, spread=30.0)
        check(z, idx, None, add, 0.01, 0.01)
        z[3, 1:] = -np.inf
        z[5] = -np.inf
        z[6, ::2] = -np.inf
        z[7] = 88.0
        z[8] = -3.0e38
        check(z, idx, None, add, 0.01, 0.01)


def test_nan_is_passed_on_and_indices_outside_are_not_counted():
    from paper_2508_02317_amd import libmoe as L
    z, idx, _, _ = make(20, 16, 2, 5)
    idx[0], idx[1] = (-1, 16), (-2 ** 31, 2 ** 31 - 1)
    z[4, 7] = np.nan
    out = L.moe_balance_loss_fwd(to_dev(z), to_dev(idx))
    assert np.array_equal(to_np(out[1]), O.balance_fwd(np.nan_to_num(z), idx)[1]) and out[0].isnan().all() and out[3][4].isnan() and out[3].isnan().sum() == 1
    g = L.moe_balance_loss_bwd(to_dev(z), out[1], out[3], 2, 1.0, 1.0)
    assert g[4].isnan().all() and g.isnan().sum() == 16


def test_no_tokens_and_the_gradient_in_place():
    import torch
    from paper_2508_02317_amd import libmoe as L
    z, idx, _, add = make(100, 24, 3, 6)
    mk = lambda n, t: torch.full((n,), 7, dtype=t, device="cuda")
    out = (mk(2, torch.float32), mk(25, torch.int32), mk(24, torch.float32), mk(0, torch.float32))
    L.moe_balance_loss_fwd(to_dev(z)[:0], to_dev(idx)[:0], out=out)
    assert not out[0].any() and not out[1].any() and not out[2].any()
    assert L.moe_balance_loss_bwd(to_dev(z)[:0], out[1], out[3], 3).shape == (0, 24)
    out = L.moe_balance_loss_fwd(to_dev(z), to_dev(idx))
    ref, g = L.moe_balance_loss_bwd(to_dev(z), out[1], out[3], 3, 0.1, 0.1, add=to_dev(add)), to_dev(add)
    assert L.moe_balance_loss_bwd(to_dev(z), out[1], out[3], 3, 0.1, 0.1, add=g, out=g) is g and torch.equal(g, ref)


def test_elements_beyond_32_bits():
    # the last rows of logits whose byte offsets pass 2^32
    import torch
    from paper_2508_02317_amd import libmoe as L
    T, E = (1 << 20) + 3, 1024
    z = torch.zeros((T, E), device="cuda")
    z[-1, 5], z[-2, 7] = 2.0, -1.0
    idx = torch.full((T, 1), 3, dtype=torch.int32, device="cuda")
    losses, counts, imp, lse = L.moe_balance_loss_fwd(z, idx)
    ref = O.balance_fwd(to_np(z[-3:]), to_np(idx[-3:]))
    tol = 40 * U * np.abs(ref[3])
    assert counts[3].item() == T and counts[E].item() == T and (np.abs(to_np(lse[-3:]) - ref[3]) <= tol).all()
    assert abs(losses[0].item() - 1.0) <= (T / 256 / 1 + 130) * U + 1e-5                 # a row or two of a million differ
    g = L.moe_balance_loss_bwd(z, counts, lse, 1, 1.0, 0.0, out=z)                       # in place of the logits
    p = ref[4]
    share = np.zeros(E)
    share[3] = E
    want = p * (share - (p @ share)[:, None]) / T
    assert (np.abs(to_np(g[-3:]) - want) <= 200 * U * p * (share + 1) / T).all()


def test_rows_taken_from_a_larger_tensor():
    # rows of an odd length that start at any multiple of four bytes
    import torch
    from paper_2508_02317_amd import libmoe as L
    for E in (13, 37, 130):
        z, idx, _, add = (None if t is None else to_dev(t) for t in make(90, E, 3, E))
        whole, more = torch.full((93, E), float("nan"), device="cuda"), torch.full((93, E), float("nan"), device="cuda")
        for first in (1, 2, 3):
            zz, aa = whole[first:first + 90], more[first:first + 90]
            zz.copy_(z)
            aa.copy_(add)
            ref, got = L.moe_balance_loss_fwd(z, idx), L.moe_balance_loss_fwd(zz, idx)
            assert all(torch.equal(p, q) for p, q in zip(ref, got))
            g = L.moe_balance_loss_bwd(z, ref[1], ref[3], 3, 0.1, 0.2, add=add)
            out = torch.full((93, E), 7.0, device="cuda")
            assert torch.equal(L.moe_balance_loss_bwd(zz, got[1], got[3], 3, 0.1, 0.2, add=aa, out=out[first:first + 90]), g)
            assert (out[:first] == 7).all() and (out[first + 90:] == 7).all()


@pytest.mark.parametrize("compiled", [True, False])
def test_both_ways_of_marshalling_and_what_they_refuse(monkeypatch, compiled):
    import torch
    from paper_2508_02317_amd import libmoe as L
    if compiled and L._marshal is None:
        pytest.skip("_marshal.so is not built here")
    z, idx, valid, add = (to_dev(t) for t in make(40, 12, 3, 7, padding=0.2))
    ref = L.moe_balance_loss_fwd(z, idx, valid)
    back = L.moe_balance_loss_bwd(z, ref[1], ref[3], 3, 0.5, 0.1, valid=valid, add=add)
    if not compiled:
        monkeypatch.setattr(L, "_marshal", None)
    assert all(torch.equal(p, q) for p, q in zip(ref, L.moe_balance_loss_fwd(z, idx, valid)))
    assert torch.equal(back, L.moe_balance_loss_bwd(z, ref[1], ref[3], 3, 0.5, 0.1, valid=valid, add=add))
    losses, counts, imp, lse = ref
    for what, call in (("float32", lambda: L.moe_balance_loss_fwd(z.double(), idx)), ("int32", lambda: L.moe_balance_loss_fwd(z, idx.long())),
                       ("topk_idx", lambda: L.moe_balance_loss_fwd(z, idx[:39])), ("valid", lambda: L.moe_balance_loss_fwd(z, idx, valid[:39])),
                       ("bool or uint8", lambda: L.moe_balance_loss_fwd(z, idx, valid.float())), ("device", lambda: L.moe_balance_loss_fwd(z, idx, valid.cpu())),
                       ("contiguous", lambda: L.moe_balance_loss_fwd(z.t(), idx)), ("counts", lambda: L.moe_balance_loss_bwd(z, counts[:12], lse, 3)),
                       ("lse", lambda: L.moe_balance_loss_bwd(z, counts, lse[:39], 3)), ("add", lambda: L.moe_balance_loss_bwd(z, counts, lse, 3, add=add[:39])),
                       ("dlosses", lambda: L.moe_balance_loss_bwd(z, counts, lse, 3, dlosses=lse)), ("losses", lambda: L.moe_balance_loss_fwd(z, idx, out=(lse, counts, imp, lse)))):
        with pytest.raises((ValueError, TypeError), match=what):
            call()
    with pytest.raises(L.MoEError, match="k=13"):
        L.moe_balance_loss_bwd(z, counts, lse, 13)
    with pytest.raises(L.MoEError, match="workspace"):
        L.moe_balance_loss_fwd(z, idx, ws=torch.empty(16, dtype=torch.uint8, device="cuda"))


def test_tokens_that_do_not_count_have_the_added_gradient_alone_whatever_the_losses_gradients_are():
    # as where a scaled loss overflows: infinities and NaN arrive in dlosses
    import torch
    from paper_2508_02317_amd import libmoe as L
    for T, E in ((40, 8), (700, 13), (300, 512)):
        z, idx, valid, add = make(T, E, 2, E, padding=0.4)
        z[3], valid[3] = -np.inf, True                                   # counts, and has no probabilities
        plain = ~valid
        plain[3] = True
        out = L.moe_balance_loss_fwd(to_dev(z), to_dev(idx), to_dev(valid))
        for dl in ((np.inf, 1.0), (1.0, -np.inf), (np.nan, np.nan)):
            for more in (add, None):
                g = to_np(L.moe_balance_loss_bwd(to_dev(z), out[1], out[3], 2, 0.1, 0.1, dlosses=to_dev(np.float32(dl)), valid=to_dev(valid), add=None if more is None else to_dev(more)))
                assert np.array_equal(g[plain], np.zeros((plain.sum(), E)) if more is None else more[plain]), (T, E, dl)
                assert not np.isfinite(g[~plain]).any(), (T, E, dl)
