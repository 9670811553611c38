"""The comparison of a layer's prompts and steps sees mistakes: each planted in the oracle is far outside the tolerance (CPU only)."""
import numpy as np
import pytest

from tests import attn_step as S


@pytest.mark.parametrize("eight_bit", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("fault", S.FAULTS)
def test_a_mistake_shows_in_every_head_of_every_sequence(fault, interleaved, eight_bit):
    window = 12 if fault == "no window" else 0
    rows, w, _, cos, sin = S.inputs(21)
    for x in rows[1:]:                                               # more than one token and more than the window
        good, bad = (S.projected(x, w, cos, sin, interleaved, eight_bit, f) for f in (None, fault))
        worst = np.zeros(S.HEADS)
        for t in range(len(x) - S.STEPS, len(x)):
            ref, tol = S.expected(*good, t, window)
            got, _ = S.expected(*bad, t, window, fault)
            worst = np.maximum(worst, (np.abs(got - ref) / tol).max(-1))
        seen = worst[1:-1] if fault == "heads in another order" else worst        # the first and the last head keep their place
        assert (seen > 8).all(), (len(x), worst)


def test_without_a_mistake_nothing_shows():
    rows, w, _, cos, sin = S.inputs(21)
    q, k, v = S.projected(rows[2], w, cos, sin, False, True)
    scores = np.einsum("hd,td->ht", q[-1][:2].astype(np.float64), k[:, 0]) / 8
    assert 1.5 < scores.std() < 4                                    # sharp, and not one token alone
    ref, tol = S.expected(q, k, v, 40, 7)
    got, _ = S.expected(q[34:41], k[34:41], v[34:41], 6, 0)
    assert np.allclose(got, ref, rtol=1e-12)
