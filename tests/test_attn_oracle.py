"""Pins of the attention oracle: formulas by hand, scalar loops, differences (CPU only)."""
import numpy as np
import pytest

from oracle import attn_oracle as A


@pytest.mark.parametrize("interleaved", [False, True])
def test_a_quarter_turn_by_hand(interleaved):
    x = np.arange(1.0, 9.0).reshape(1, 1, 8)
    cos, sin = np.array([[0.0, 1.0]]), np.array([[1.0, 0.0]])        # the first pair a quarter, the second not at all; rot = 4
    y = A.rope(x, cos, sin, interleaved)[0, 0]
    assert y.tolist() == ([-2, 1, 3, 4, 5, 6, 7, 8] if interleaved else [-3, 2, 1, 4, 5, 6, 7, 8])
    back = A.rope(y.reshape(1, 1, 8), cos, sin, interleaved, back=True)
    assert np.array_equal(back, x)


@pytest.mark.parametrize("interleaved", [False, True])
def test_scores_of_turned_heads_depend_on_distance_alone(interleaved):
    r = np.random.default_rng(0)
    cos, sin = A.rope_table(10000.0 ** (-np.arange(0, 16, 2) / 16), 40)
    q, k = r.standard_normal((1, 1, 16)), r.standard_normal((1, 1, 16))
    at = lambda x, p: A.rope(x, cos[p:p + 1], sin[p:p + 1], interleaved)[0, 0]
    assert abs(at(q, 7) @ at(k, 3) - at(q, 39) @ at(k, 35)) < 1e-12


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot", [16, 32])
def test_the_gradient_against_differences(interleaved, rot):
    r = np.random.default_rng(1)
    x, g = r.standard_normal((3, 2, 32)), r.standard_normal((3, 2, 32))
    cos, sin = A.rope_table(np.exp(-np.arange(rot // 2)), 3)
    dx, h = A.rope(g, cos, sin, interleaved, back=True), 1e-6
    for i in np.ndindex(*x.shape):
        e = np.zeros_like(x)
        e[i] = h
        d = ((A.rope(x + e, cos, sin, interleaved) - A.rope(x - e, cos, sin, interleaved)) * g).sum() / (2 * h)
        assert abs(d - dx[i]) < 1e-8


def test_attention_against_scalar_loops():
    r = np.random.default_rng(2)
    q, k, v = r.standard_normal((4, 8)), r.standard_normal((5, 2, 8)), r.standard_normal((5, 2, 8))
    out, lse, _, _ = A.attend(q, k, v, 0.3)
    for h in range(4):
        e = [np.exp(0.3 * sum(q[h, d] * k[t, h // 2, d] for d in range(8))) for t in range(5)]
        assert abs(lse[h] - np.log(sum(e))) < 1e-12
        for d in range(8):
            assert abs(out[h, d] - sum(e[t] * v[t, h // 2, d] for t in range(5)) / sum(e)) < 1e-12
    out, lse, _, _ = A.attend(q, k[:0], v[:0], 0.3)
    assert not out.any() and np.all(lse == -np.inf)


def test_tokens_are_found_through_their_pages():
    cache = np.arange(4 * 1 * 16 * 2, dtype=np.float64).reshape(4, 1, 16, 2)
    rows = A.gather(cache, None, [2, 0], 16, 14, 4)
    assert np.array_equal(rows[:, 0], np.concatenate([cache[2, 0, 14:], cache[0, 0, :2]]))
