"""The oracle of the norm, of positions with several axes and of the router's losses against hand-made values, independent forms and central differences
(CPU only)."""
import numpy as np
import pytest

from oracle import attn_oracle as A
from oracle import train_oracle as O


def test_norm_by_hand():
    y, m, r = O.norm([[1.0, 3.0], [-2.0, -2.0]], eps=0.25)
    assert m.tolist() == [2.0, -2.0] and np.allclose(r, [1.25 ** -0.5, 2.0]) and np.allclose(y, [[-1.25 ** -0.5, 1.25 ** -0.5], [0, 0]])
    y, m, r = O.norm([[3.0, 4.0]], weight=[2.0, 1.0], bias=[0.0, 1.0], eps=0.0, rms=True)
    assert m.tolist() == [0.0] and np.allclose(r, 12.5 ** -0.5) and np.allclose(y, [[6 / 12.5 ** 0.5, 4 / 12.5 ** 0.5 + 1]])


def _difference(f, x, step=1e-5):
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        up, down = x.copy(), x.copy()
        up[i] += step
        down[i] -= step
        g[i] = (f(up) - f(down)) / (2 * step)
    return g


@pytest.mark.parametrize("rms", [False, True])
def test_norm_gradients_are_differences(rms):
    r = np.random.default_rng(3)
    x, dy, add, w, b = r.standard_normal((3, 2, 8)), r.standard_normal((3, 2, 8)), r.standard_normal((3, 2, 8)), 1 + r.standard_normal(8), r.standard_normal(8)
    _, m, rstd = O.norm(x, w, b, 0.1, rms)
    dx, dw, db = O.norm_bwd(dy, x, m, rstd, w, add, rms)
    loss = lambda x, w, b: (dy * O.norm(x, w, b, 0.1, rms)[0]).sum()
    assert np.allclose(dx - add, _difference(lambda v: loss(v, w, b), x), atol=1e-8)
    assert np.allclose(dw, _difference(lambda v: loss(x, v, b), w), atol=1e-8) and np.allclose(db, _difference(lambda v: loss(x, w, v), b), atol=1e-8)


def test_axes_with_equal_positions_are_one_axis_and_pairs_go_by_their_own():
    r = np.random.default_rng(1)
    x, pos, axis = r.standard_normal((5, 2, 16)), r.integers(0, 9, (3, 5)), [0, 0, 1, 1, 1, 2, 2, 0]
    cos, sin = A.rope_table(10.0 ** -np.arange(8), 9)
    same = np.repeat(pos[:1], 3, axis=0)
    assert np.array_equal(O.rope_axes(x, cos, sin, same, axis, False), A.rope(x, cos[pos[0]], sin[pos[0]], False))
    y = O.rope_axes(x, cos, sin, pos, axis, False)
    for t in range(5):
        for i, a in enumerate(axis):
            c, s = np.cos(pos[a, t] * 10.0 ** -i), np.sin(pos[a, t] * 10.0 ** -i)
            assert np.allclose(y[t, :, i], x[t, :, i] * c - x[t, :, i + 8] * s) and np.allclose(y[t, :, i + 8], x[t, :, i + 8] * c + x[t, :, i] * s)
    assert np.allclose(O.rope_axes(y, cos, sin, pos, axis, False, back=True), x)


def test_balance_by_hand_and_at_its_least():
    # two tokens, two experts, one choice each, probabilities 3/4 and 1/4
    z = np.log([[3.0, 1.0], [3.0, 1.0]])
    losses, counts, imp, lse, _ = O.balance_fwd(z, [[0], [1]])
    assert counts.tolist() == [1, 1, 2] and np.allclose(imp, [0.75, 0.25]) and np.allclose(losses, [2 / 2 * 1.0, np.log(4) ** 2]) and np.allclose(lse, np.log(4))
    losses, counts, _, _, _ = O.balance_fwd(z, [[0], [0]])
    assert counts.tolist() == [2, 0, 2] and np.isclose(losses[0], 1.5)
    losses, counts, imp, _, _ = O.balance_fwd(np.zeros((4, 2)), [[0], [1], [0], [1]], [1, 1, 0, 0])
    assert counts.tolist() == [1, 1, 2] and np.isclose(losses[0], 1.0) and np.allclose(imp, 0.5)
    losses, counts, imp, lse, _ = O.balance_fwd(z, [[0], [0]], [0, 0])
    assert losses.tolist() == [0, 0] and counts.tolist() == [0, 0, 0] and imp.tolist() == [0, 0] and lse.tolist() == [0, 0]


def test_balance_gradient_is_the_difference():
    r = np.random.default_rng(5)
    z, valid = r.standard_normal((6, 5)), np.array([1, 0, 1, 1, 1, 0])
    idx = np.argsort(-z, axis=1)[:, :2]
    f = lambda v: O.balance_fwd(v, idx, valid)[0] @ [0.7, 0.3]
    assert np.allclose(O.balance_bwd(z, idx, 0.7, 0.3, valid), _difference(f, z), atol=1e-8)
    assert np.allclose(O.balance_bwd(z, idx, 0.7, 0.0).sum(1), 0)         # probabilities sum to 1 whatever the logits


def test_logits_of_minus_infinity_have_no_part():
    z = np.array([[0.0, -np.inf, 1.0], [-np.inf] * 3, [0.5, 0.5, 0.5]])
    idx = np.array([[2], [0], [1]])
    losses, counts, imp, lse, p = O.balance_fwd(z, idx)
    assert np.isfinite(losses).all() and lse[1] == -np.inf and p[0, 1] == 0 and p[1].tolist() == [0, 0, 0] and counts.tolist() == [1, 1, 1, 3]
    assert np.isfinite(O.balance_bwd(z, idx, 1.0, 1.0)).all() and not O.balance_bwd(z, idx, 1.0, 1.0)[1].any()
