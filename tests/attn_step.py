"""Prompts and steps of one attention layer whose projections are exact, and their expected outputs (test infrastructure only).

Rows and weights are small integers times powers of two, so that a projection's products and sums are exact in fp32 in any order and its result is
rounded once, to bf16; the output projection is the identity.  The rotation's products and sums are rounded one by one in fp32, which numpy repeats,
and blocks of 8 bits are formed from that.  So keys, values and queries are known bit for bit, and what is left is the attention itself.
Queries and keys are large enough that scores spread over several units and every head looks at few of its tokens."""
import numpy as np

from oracle import attn_oracle as A
from oracle import moe_fp8 as F
from tests.util import q as rounded

HEADS, KV_HEADS, DIM, N_POS = 4, 2, 64, 128
D = HEADS * DIM
LENGTHS, STEPS = (1, 17, 40, 64), 6


def inputs(seed):
    """Rows [n, D] of every sequence (prompt and steps), w_qkv [(HEADS + 2 KV_HEADS) DIM, D], w_out [D, D], cos and sin [N_POS, DIM / 2], all float32."""
    r = np.random.default_rng(seed)
    rows = [r.integers(-3, 4, (n + STEPS, D)).astype(np.float32) for n in LENGTHS]
    w = r.integers(-7, 8, ((HEADS + 2 * KV_HEADS) * DIM, D)).astype(np.float32) / 64
    w[HEADS * DIM:(HEADS + KV_HEADS) * DIM] /= 2
    cos, sin = (x.astype(np.float32) for x in A.rope_table(10000.0 ** (-np.arange(0, DIM, 2) / DIM), N_POS))
    return rows, w, np.eye(D, dtype=np.float32), cos, sin


def projected(rows, w, cos, sin, interleaved, eight_bit, fault=None):
    """q [n, HEADS, DIM], k, v [n, KV_HEADS, DIM] of one sequence as the layer holds them."""
    exact = rows.astype(np.float64) @ w.astype(np.float64).T
    assert np.array_equal(exact * 64 * 2, np.round(exact * 64 * 2)) and np.abs(exact).max() * 128 < 2 ** 24
    q, k, v = np.split(rounded(exact, "bf16").reshape(len(rows), -1, DIM), [HEADS, HEADS + KV_HEADS], axis=1)
    c, s = cos[:len(rows)], sin[:len(rows)]
    turn = lambda x, back=False, layout=interleaved: A.rope(x, c, s, layout, back, dtype=np.float32)
    other = not interleaved if fault == "wrong pairs" else interleaved
    qr = q if fault in ("no rotation", "queries not rotated") else turn(q, layout=other)
    kr = k if fault == "no rotation" else turn(k, back=fault == "keys rotated backwards", layout=other)
    qr = rounded(qr, "bf16")
    if eight_bit:
        return qr, F.mx_dequantise(*F.mx_quantise(kr)), F.mx_dequantise(*F.mx_quantise(v))
    return qr, rounded(kr, "bf16").astype(np.float64), v.astype(np.float64)


def expected(q, k, v, t, window, fault=None):
    """Token t's output [HEADS, DIM] in float64, and how far a result may be from it (as derived for the attention of one token over bf16 or 8 bits)."""
    lo = max(0, t + 1 - window) if window and fault != "no window" else 0
    hi = t if fault == "own key missing" and t > lo else t + 1
    scale = 0.0 if fault == "scores ignored" else 1.0 if fault == "no scale" else DIM ** -0.5
    qt = q[t]
    if fault == "heads in another order":
        qt = qt.reshape(HEADS // KV_HEADS, KV_HEADS, DIM).transpose(1, 0, 2).reshape(HEADS, DIM)
    out, _, bound, top = A.attend(qt, k[lo:hi], v[lo:hi], scale)
    if fault == "heads in another order":
        out = out.reshape(KV_HEADS, HEADS // KV_HEADS, DIM).transpose(1, 0, 2).reshape(HEADS, DIM)
    eps = (DIM + 4) * 2.0 ** -24 * top + 2.0 ** -22 * top + 2.0 ** -22 + 2.0 ** -16 + ((hi - lo) / 16 + 64) * 2.0 ** -24
    tol = 2 * eps[:, None] * bound
    return out, tol + A.half_place(np.abs(out) + tol, 8)


FAULTS = ["no rotation", "wrong pairs", "keys rotated backwards", "queries not rotated", "scores ignored", "own key missing", "no window", "no scale",
          "heads in another order"]
