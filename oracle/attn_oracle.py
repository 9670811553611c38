"""fp64 CPU oracle for rotary positions, the paged key/value cache and the attention of one token over it.

TEST INFRASTRUCTURE ONLY.  Nothing in the product path may import this module; it shares no code,
table or constant with the HIP path.  8-bit blocks are those of oracle/moe_fp8.py.
"""
import numpy as np

from . import moe_fp8 as F


def rope_table(freq, n_pos, amplitude=1.0):
    """Angles in extended precision, reduced and evaluated there: cos, sin [n_pos, half] as float64."""
    a = np.arange(n_pos, dtype=np.longdouble)[:, None] * np.asarray(freq, dtype=np.longdouble)
    return (np.cos(a) * amplitude).astype(np.float64), (np.sin(a) * amplitude).astype(np.float64)


def pairs(D, rot, interleaved):
    """(index of a, index of b) of every pair."""
    i = np.arange(rot // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)


def rope(x, cos, sin, interleaved, back=False, dtype=np.float64):
    """x [T, H, D] turned; cos, sin [T, rot/2] of its tokens.  dtype float32: every product and sum rounded there, one by one."""
    x, c, s = np.asarray(x).astype(dtype), np.asarray(cos).astype(dtype)[:, None], np.asarray(sin).astype(dtype)[:, None]
    if back:
        s = -s
    ia, ib = pairs(x.shape[2], 2 * c.shape[2], interleaved)
    a, b, y = x[..., ia], x[..., ib], x.copy()
    y[..., ia] = a * c - b * s
    y[..., ib] = b * c + a * s
    return y


def rope_magnitude(x, cos, sin, interleaved):
    """|a c| + |b s| of every output element (what its rounding errors go by); 0 where nothing is turned."""
    x, c, s = np.abs(np.asarray(x, dtype=np.float64)), np.abs(np.asarray(cos, dtype=np.float64))[:, None], np.abs(np.asarray(sin, dtype=np.float64))[:, None]
    ia, ib = pairs(x.shape[2], 2 * c.shape[2], interleaved)
    m = np.zeros_like(x)
    m[..., ia] = x[..., ia] * c + x[..., ib] * s
    m[..., ib] = x[..., ib] * c + x[..., ia] * s
    return m


def half_place(x, bits):
    """Half a unit in the last of `bits` places of x > 0 (8: bfloat16, 24: float32): the most that rounding to nearest changes it by."""
    _, e = np.frexp(x)                                 # x = m 2^e, 1/2 <= m < 1
    return np.exp2(np.asarray(e, dtype=np.float64) - bits - 1)


def gather(cache, scales, block_table_row, page_size, first, count):
    """Tokens first .. first + count - 1 of one sequence, one by one: [count, heads, dim] float64."""
    rows = []
    for t in range(first, first + count):
        page, at = int(block_table_row[t // page_size]), t % page_size
        row = cache[page, :, at]
        rows.append(F.mx_dequantise(row, scales[page, :, at]) if scales is not None else row.astype(np.float64))
    return np.stack(rows) if rows else np.zeros((0, cache.shape[1], cache.shape[3]))


def attend(q, k, v, scale):
    """q [Hq, D], k, v [L, H, D] -> out [Hq, D], lse [Hq], bound [Hq, D] = sum p |v|, top [Hq] = max_t sum |q k| |scale|."""
    Hq, D = q.shape
    L, H, _ = k.shape
    if L == 0:
        return np.zeros((Hq, D)), np.full(Hq, -np.inf), np.zeros((Hq, D)), np.zeros(Hq)
    q = q.astype(np.float64)
    out, lse, bound, top = np.zeros((Hq, D)), np.zeros(Hq), np.zeros((Hq, D)), np.zeros(Hq)
    for h in range(Hq):
        kk, vv = k[:, h // (Hq // H)], v[:, h // (Hq // H)]
        s = scale * (kk @ q[h])
        m = s.max()
        p = np.exp(s - m)
        total = p.sum()
        out[h], lse[h], bound[h] = p @ vv / total, m + np.log(total), p @ np.abs(vv) / total
        top[h] = abs(scale) * (np.abs(kk) @ np.abs(q[h])).max()
    return out, lse, bound, top
