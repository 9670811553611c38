"""fp64 CPU oracle for the norm, rotary positions with several axes and the router's losses.

TEST INFRASTRUCTURE ONLY.  Nothing in the product path may import this module; it shares no code,
table or constant with the HIP path.
"""
import numpy as np

from . import attn_oracle as A


def norm(h, weight=None, bias=None, eps=1e-6, rms=False):
    """Rows of h [..., D] -> y, mean (zeros with rms), rstd."""
    h = np.asarray(h, dtype=np.float64)
    mean = np.zeros(h.shape[:-1]) if rms else h.mean(-1)
    c = h - mean[..., None]
    rstd = 1.0 / np.sqrt((c * c).mean(-1) + eps)
    y = c * rstd[..., None]
    y = y if weight is None else y * np.asarray(weight, dtype=np.float64)
    return (y if bias is None else y + np.asarray(bias, dtype=np.float64)), mean, rstd


def norm_bwd(dy, h, mean, rstd, weight=None, add=None, rms=False):
    """-> dx, dweight, dbias of the rows that mean and rstd belong to."""
    dy, h = np.asarray(dy, dtype=np.float64), np.asarray(h, dtype=np.float64)
    r = np.asarray(rstd, dtype=np.float64)[..., None]
    xh = (h if rms else h - np.asarray(mean, dtype=np.float64)[..., None]) * r
    g = dy if weight is None else dy * np.asarray(weight, dtype=np.float64)
    dx = g - xh * (g * xh).mean(-1, keepdims=True)
    if not rms:
        dx = dx - g.mean(-1, keepdims=True)
    dx = dx * r
    if add is not None:
        dx = dx + np.asarray(add, dtype=np.float64)
    rows = tuple(range(h.ndim - 1))
    return dx, (dy * xh).sum(rows), dy.sum(rows)


def axes_table(table, positions, pair_axis):
    """table [n_pos, half], positions [axes, T] -> [T, half]: each pair's column at the position of its axis (clamped into the table)."""
    table, positions = np.asarray(table), np.clip(np.asarray(positions), 0, len(table) - 1)
    return np.stack([table[positions[a], i] for i, a in enumerate(pair_axis)], axis=1) if len(pair_axis) else table[:0, :0]


def rope_axes(x, cos, sin, positions, pair_axis, interleaved, back=False):
    return A.rope(x, axes_table(cos, positions, pair_axis), axes_table(sin, positions, pair_axis), interleaved, back)


def balance_fwd(logits, topk_idx, valid=None):
    """-> losses [2], counts [E + 1], importance [E], lse [T], p [T, E] (zeros for tokens that are not valid)."""
    z, idx = np.asarray(logits, dtype=np.float64), np.asarray(topk_idx)
    (T, E), k = z.shape, idx.shape[1]
    ok = np.ones(T, dtype=bool) if valid is None else np.asarray(valid).astype(bool)
    n = int(ok.sum())
    p, lse = np.zeros((T, E)), np.zeros(T)
    for t in np.flatnonzero(ok):
        top = z[t].max()
        if top == -np.inf:
            lse[t] = -np.inf
            continue
        e = np.exp(z[t] - top)
        p[t], lse[t] = e / e.sum(), top + np.log(e.sum())
    chosen = idx[ok].ravel()
    counts = np.bincount(chosen[(chosen >= 0) & (chosen < E)], minlength=E)
    many = max(n, 1)
    importance = p.sum(0) / many
    finite = lse[ok][lse[ok] > -np.inf]
    losses = np.array([E / (k * many) * (counts * importance).sum(), (finite ** 2).sum() / many])
    return losses, np.concatenate((counts, [n])), importance, lse, p


def balance_bwd(logits, topk_idx, balance, z_weight, valid=None, add=None):
    _, counts, _, lse, p = balance_fwd(logits, topk_idx, valid)
    E, k, n = p.shape[1], np.asarray(topk_idx).shape[1], max(int(counts[-1]), 1)
    share = counts[:E] * E / (k * n)
    lse = np.where(lse == -np.inf, 0.0, lse)
    d = p * (balance / n * (share - (p @ share)[:, None]) + z_weight * 2 / n * lse[:, None])
    return d if add is None else d + np.asarray(add, dtype=np.float64)
