"""Workloads of what a training step of a block for text, images and video has around attention and experts: the norm in front of each half,
rotary positions with several axes, and the loss that keeps the router balanced.

A case is a dict of sizes and options.  `prepare` makes what a program holds before the call, `run` is one pass, `exact` the same in 64 bits, `work`
the bytes and operations a pass cannot do without.  With `own` false `run` uses elementary torch operations in 32 bits; with `own` true the
library's entry points.

Kinds (`op`):
  norm     rows of `dim` elements, `heads` of them a token: layer norm or rms norm of x, or of x + residual, which is returned too; with
           `back` the gradients of input, weight and bias, with `residual` added to that of the input
  axes     queries and keys turned by positions that have several axes (time, height, width); each pair of a head's elements belongs to one of
           them.  `layout` says which: "sections" of the pairs (a quarter and two equal parts for three axes), "uneven" ones, or "cycled";
           with `back` the gradients, with `store` keys and values go into the pages of a cache in the same call
  balance  the router's balance loss and z loss over the tokens that are not padding, with the counts per expert, and the gradient of their
           weighted sum; with `residual` added to the logits' gradient from the experts
"""
import math
import random

import torch

own = False

_DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
_BASE = 1e6                                            # base of the rotation's frequencies
_PAGE = 64
_WEIGHTS = (0.01, 0.001)                               # of balance loss and z loss in the sum whose gradient is taken


def _case(op, **options):
    c = dict(op=op, tokens=0, heads=1, dim=128, dtype="bf16", back=False, rms=True, residual=False, bias=False, weights="f32", fused=False, kv_heads=0, rot=0,
             interleaved=False, axes=0, layout="sections", positions=0, store=False, experts=0, k=0, padding=0.0)
    c.update(options)
    return c


def listed():
    cases = {
        # one generation step of 16 sequences: the residual stream between attention and experts
        "norm_16": _case("norm", tokens=16, dim=2048, residual=True),
        # the same for one 8K-token micro-batch of training
        "norm_8k": _case("norm", tokens=8192, dim=2048, residual=True),
        # gradients of the query norm of that micro-batch, the queries being a view of one projection's output
        "norm_8k_heads_back": _case("norm", tokens=8192, heads=32, dim=128, back=True, fused=True),
        # gradients of one sequence shard of a 160K-token sequence, the residual stream's gradient coming in
        "norm_40k_back": _case("norm", tokens=40960, dim=2048, back=True, residual=True, weights="bf16"),
        # layer norm of an image encoder in full precision: an odd number of patches, a row that is no power of two
        "norm_odd_layer_f32_back": _case("norm", tokens=1531, dim=1000, dtype="f32", rms=False, bias=True, back=True),
        # one generation step: the new token of every sequence is rotated and stored
        "axes_16_store": _case("axes", tokens=16, heads=32, kv_heads=4, rot=128, axes=3, positions=2000, fused=True, store=True),
        # an 8K-token micro-batch of text, images and video
        "axes_8k": _case("axes", tokens=8192, heads=32, kv_heads=4, rot=128, axes=3, fused=True),
        # gradients of one shard of a long video, the axes taking turns over the pairs
        "axes_40k_cycled_back": _case("axes", tokens=40960, heads=32, kv_heads=4, rot=128, axes=3, layout="cycled", back=True, positions=60000),
        # patches of an image encoder, two axes, in full precision
        "axes_odd_patches_f32": _case("axes", tokens=1531, heads=16, kv_heads=16, dim=64, rot=64, axes=2, dtype="f32"),
        # a full-precision parity run: few tokens, few experts
        "balance_256": _case("balance", tokens=256, experts=8, k=2),
        # the router of one 8K-token micro-batch
        "balance_8k": _case("balance", tokens=8192, experts=128, k=8, residual=True),
        # a shard of a long sequence, its tail padding
        "balance_40k_padded": _case("balance", tokens=40960, experts=128, k=8, residual=True, padding=0.1),
    }
    return [dict(c, name=n) for n, c in cases.items()]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm", "axes", "axes", "balance", "balance"])
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    tokens = _log_int(rng, 1, 40960)
    if op == "norm":
        rms = rng.random() < 0.6
        c = _case(op, tokens=tokens, dtype=dtype, rms=rms, back=rng.random() < 0.5, bias=not rms and rng.random() < 0.8, weights=rng.choice(["f32", dtype]))
        if rng.random() < 0.3:                         # of queries or keys
            c.update(heads=rng.choice([1, 2, 4, 8, 16, 28, 32]), dim=rng.choice([64, 128, 192, 256]), fused=rng.random() < 0.5)
        else:
            c.update(dim=8 * _log_int(rng, 8, 1024), residual=rng.random() < 0.6)
    elif op == "axes":
        dim, kv_heads = rng.choice([64, 128, 128, 192, 256]), rng.choice([1, 2, 4, 8])
        c = _case(op, tokens=tokens, dtype=dtype, dim=dim, kv_heads=kv_heads, heads=kv_heads * rng.choice([1, 2, 4, 7, 8]), rot=rng.choice([dim, dim, dim // 2]),
                  interleaved=rng.random() < 0.3, axes=rng.choice([2, 3, 3, 4]), layout=rng.choice(["sections", "uneven", "cycled"]),
                  positions=rng.choice([0, 0, 2000, 60000]), fused=rng.random() < 0.5)
        c.update(rng.choice([{}, {"back": True}, {"store": True}]))
    else:
        experts = _log_int(rng, 2, 1024)
        c = _case(op, tokens=tokens, experts=experts, k=rng.randint(1, min(experts, 16)), padding=rng.choice([0.0, 0.0, 0.05, 0.5]), residual=rng.random() < 0.6)
    most = 0.9 * max(work(big)["bytes"] for big in listed())
    while work(c)["bytes"] > most:
        c["tokens"] = (c["tokens"] + 1) // 2
    return c


def work(case):
    c = case
    T, es = c["tokens"], 4 if c["dtype"] == "f32" else 2
    if c["op"] == "norm":
        rows, moved, vector = T * c["heads"], T * c["heads"] * c["dim"] * es, c["dim"] * (4 if c["weights"] == "f32" else 2)
        stats = 4 * rows * (1 if c["rms"] else 2)
        # forward: x, residual, their sum, y; backward: x, dy, residual, dx
        passes = (3 if c["back"] else 2) + (c["residual"] and (1 if c["back"] else 2))
        vectors = (3 if c["back"] else 2) * vector if c["bias"] else (2 if c["back"] else 1) * vector
        return {"bytes": passes * moved + stats + vectors, "flops": rows * c["dim"] * (12 if c["back"] else 7)}
    if c["op"] == "axes":
        q, kv = c["heads"] * c["dim"] * es, c["kv_heads"] * c["dim"] * es
        table = c["rot"] * 4 + 4 * c["axes"]           # cosines and sines of a token's pairs, its positions
        store = (2 * kv + 8) if c["store"] else 0
        return {"bytes": T * (2 * (q + kv) + table + store), "flops": T * 3 * c["rot"] * (c["heads"] + c["kv_heads"])}
    pairs, E = T * c["k"], c["experts"]
    mask = T if c["padding"] else 0
    return {"bytes": (3 if c["residual"] else 2) * 4 * T * E + 4 * pairs + mask + 4 * T + 8 * E, "flops": 14 * T * E}


# ---- inputs -----------------------------------------------------------------------------------------------

def _normal(gen, shape, std, dtype):
    return (torch.randn(shape, generator=gen, device="cuda") * std).to(dtype)


def _heads(gen, c, rows, groups):
    """[rows, h, dim] for each h of `groups`: tensors of their own, or views of one projection's output."""
    d, dtype = c["dim"], _DTYPE[c["dtype"]]
    if not c["fused"]:
        return [_normal(gen, (rows, h, d), 1.0, dtype) for h in groups]
    return list(_normal(gen, (rows, sum(groups), d), 1.0, dtype).split(groups, dim=1))


def _pair_axis(c):
    """The axis of every pair of a head's elements."""
    half, A = c["rot"] // 2, c["axes"]
    if c["layout"] == "cycled":
        return [i % A for i in range(half)]
    sizes = {2: [half // 2], 3: [half // 4, (half - half // 4) // 2], 4: [half // 4] * 3}[A]
    if c["layout"] == "uneven":
        sizes = [n + 3 - 2 * i for i, n in enumerate(sizes)]
    sizes.append(half - sum(sizes))
    return [a for a, n in enumerate(sizes) for _ in range(n)]


def _positions(c, seed):
    """Positions [axes, tokens] of runs of text, images and video: all axes go on together over text; over a picture the first stays where it is, or
    counts the frames, and the others are row and column; what follows begins behind the largest of them."""
    rng, A, left, at, parts = random.Random(seed), c["axes"], c["tokens"], c["positions"], []
    while left > 0:
        if A > 2 and rng.random() < 0.5:
            n = min(left, rng.randint(8, 512))
            parts.append((torch.arange(n, dtype=torch.int32) + at).expand(A, n))
            at += n
        else:
            frames, rows, cols = rng.choice([1, 1, 4]) if A > 2 else 1, rng.randint(4, 32), rng.randint(4, 32)
            n = min(left, frames * rows * cols)
            grid = torch.stack(torch.meshgrid(*(torch.arange(m, dtype=torch.int32) for m in (frames, rows, cols)), indexing="ij")).view(3, -1)[:, :n] + at
            parts.append({2: grid[1:], 3: grid, 4: torch.cat((grid, torch.full((1, n), at, dtype=torch.int32)))}[A])
            at += max(frames, rows, cols) if A > 2 else 0
        left -= n
    return torch.cat(parts, dim=1)


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    s, dtype, T, d = {"case": c}, _DTYPE[c["dtype"]], c["tokens"], c["dim"]
    empty = lambda shape, t: torch.empty(shape, dtype=t, device="cuda")
    if c["op"] == "norm":
        shape, wt = (T, c["heads"], d), _DTYPE[c["weights"]]
        # hidden states: a few large channels, rows of different size, an offset where there is a mean to take off
        channel = torch.exp(0.5 * torch.randn(d, generator=gen, device="cuda"))
        row = torch.exp(0.5 * torch.randn((T, 1, 1), generator=gen, device="cuda"))
        wide = _heads(gen, dict(c, dtype="f32"), T, [c["heads"], 4])[0] if c["fused"] else torch.randn(shape, generator=gen, device="cuda")
        x = wide.mul_(channel).mul_(row)
        if not c["rms"]:
            x += 0.5 * row
        if c["fused"]:                                 # the view of a wider tensor, in the type of the case
            wide = empty((T, c["heads"] + 4, d), dtype)
            wide[:, :c["heads"]], x = x, wide[:, :c["heads"]]
        else:
            x = x.to(dtype)
        s["x"] = x if c["heads"] > 1 else x[:, 0]
        s["weight"] = (1 + 0.1 * torch.randn(d, generator=gen, device="cuda")).to(wt)
        s["bias"] = (0.1 * torch.randn(d, generator=gen, device="cuda")).to(wt) if c["bias"] else None
        s["residual"] = _normal(gen, s["x"].shape, 1.0, dtype) if c["residual"] else None
        if c["back"]:
            s["dy"] = _normal(gen, s["x"].shape, 1.0, dtype)
            x64 = s["x"].double()                      # what the forward pass kept of each row
            m = None if c["rms"] else x64.mean(-1)
            v = x64.square().mean(-1) if c["rms"] else (x64 - m[..., None]).square().mean(-1)
            s["mean"], s["rstd"] = None if c["rms"] else m.float(), (v + 1e-6).rsqrt().float()
        if own:
            from paper_2508_02317_amd import libmoe as L
            rows = s["x"].shape[:-1]
            if c["back"]:
                s["out"] = (empty(s["x"].shape, dtype), empty(d, wt), empty(d, wt) if c["bias"] else None)
                s["ws"] = empty(L.lib.moe_norm_bwd_workspace_bytes(T, c["heads"], d), torch.uint8)
            else:
                s["out"] = (empty(s["x"].shape, dtype), empty(s["x"].shape, dtype) if c["residual"] else None,
                            None if c["rms"] else empty(rows, torch.float32), empty(rows, torch.float32))
    elif c["op"] == "axes":
        s["pair_axis"] = bytes(_pair_axis(c))
        s["positions"] = _positions(c, seed).cuda().contiguous()
        angle = torch.arange(c["positions"] + T + 64, dtype=torch.float64, device="cuda")[:, None] * _BASE ** (
            -torch.arange(0, c["rot"], 2, dtype=torch.float64, device="cuda") / c["rot"])
        s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
        kvh = c["kv_heads"]
        if c["store"]:
            s["q"], s["k"], s["v"] = _heads(gen, c, T, [c["heads"], kvh, kvh])
            pages = -(-T // _PAGE) + 3
            s["kc"], s["vc"] = (_normal(gen, (pages, kvh, _PAGE, d), 1.0, dtype) for _ in range(2))
            s["slots"] = torch.randperm(pages * _PAGE, generator=gen, device="cuda")[:T] if T <= 64 else torch.arange(T, device="cuda") + _PAGE
        else:
            s["q"], s["k"] = _heads(gen, c, T, [c["heads"], kvh])
        if own:
            from paper_2508_02317_amd import libmoe as L
            s["out"] = (empty((T, c["heads"], d), dtype), empty((T, kvh, d), dtype))
            if c["store"]:
                s["cache"] = L.moe_kv_cache(s["kc"], s["vc"])
    else:
        E, k = c["experts"], c["k"]
        # some experts are asked for more often than others
        s["logits"] = 1.5 * torch.randn((T, E), generator=gen, device="cuda") + 0.7 * torch.randn(E, generator=gen, device="cuda")
        s["topk_idx"] = s["logits"].topk(k, dim=1).indices.int().contiguous()
        # the experts' part of a mean loss' gradient
        s["add"] = 1e-4 / T * torch.randn((T, E), generator=gen, device="cuda") if c["residual"] else None
        s["valid"] = None
        if c["padding"]:                               # sequences of a padded batch: each ends in padding
            n = max(1, T // 8)
            s["valid"] = torch.arange(T, device="cuda") % n < n * (1 - c["padding"])
        if own:
            from paper_2508_02317_amd import libmoe as L
            s["fwd"] = (empty(2, torch.float32), empty(E + 1, torch.int32), empty(E, torch.float32), empty(T, torch.float32))
            s["dlogits"] = empty((T, E), torch.float32)
            s["ws"] = empty(L.lib.moe_balance_loss_fwd_workspace_bytes(T, E, k), torch.uint8)
    return s


# ---- the plain forms --------------------------------------------------------------------------------------

def _plain_norm(s):
    c, dtype = s["case"], s["x"].dtype
    w = s["weight"].float()
    if not c["back"]:
        out = {}
        h = s["x"].float()
        if c["residual"]:
            out["h"] = (h + s["residual"].float()).to(dtype)
            h = out["h"].float()
        if not c["rms"]:
            out["mean"] = h.mean(-1)
            h = h - out["mean"][..., None]
        out["rstd"] = 1 / (h.square().mean(-1) + 1e-6).sqrt()
        y = h * out["rstd"][..., None] * w
        out["y"] = (y + s["bias"].float() if c["bias"] else y).to(dtype)
        return out
    r, dy = s["rstd"][..., None], s["dy"].float()
    xh = (s["x"].float() if c["rms"] else s["x"].float() - s["mean"][..., None]) * r
    g = dy * w
    dx = g - xh * (g * xh).mean(-1, keepdim=True)
    if not c["rms"]:
        dx = dx - g.mean(-1, keepdim=True)
    dx = dx * r
    if c["residual"]:
        dx = dx + s["residual"].float()
    rows = tuple(range(dy.dim() - 1))
    out = {"dx": dx.to(dtype), "dweight": (dy * xh).sum(rows).to(s["weight"].dtype)}
    if c["bias"]:
        out["dbias"] = dy.sum(rows).to(s["weight"].dtype)
    return out


def _turn(x, cos, sin, interleaved):
    """x [T, h, d] rotated, in 32 bits; cos and sin [T, rot / 2]."""
    rot = 2 * cos.shape[1]
    x, cos, sin = x.float(), cos[:, None], sin[:, None]
    if interleaved:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y = torch.stack((a * cos - b * sin, b * cos + a * sin), dim=-1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y = torch.cat((a * cos - b * sin, b * cos + a * sin), dim=-1)
    return torch.cat((y, x[..., rot:]), dim=-1)


def _plain_axes(s):
    c = s["case"]
    pair = torch.arange(c["rot"] // 2, device="cuda")
    at = s["positions"][torch.tensor(list(s["pair_axis"])).cuda()].long().t()                        # [T, rot / 2]
    cos, sin = s["cos"][at, pair], s["sin"][at, pair]
    sin = -sin if c["back"] else sin
    q, k = (_turn(s[n], cos, sin, c["interleaved"]).to(s[n].dtype) for n in "qk")
    if not c["store"]:
        return {"q": q, "k": k}
    page, place = s["slots"] // _PAGE, s["slots"] % _PAGE
    s["kc"][page, :, place], s["vc"][page, :, place] = k, s["v"]
    return {"q": q, "k_cache": s["kc"], "v_cache": s["vc"]}


def _plain_balance(s):
    c, z = s["case"], s["logits"]
    T, E = z.shape
    valid = s["valid"] if s["valid"] is not None else torch.ones(T, dtype=torch.bool, device="cuda")
    top = z.amax(1, keepdim=True)
    e = (z - top).exp()
    total = e.sum(1, keepdim=True)
    lse = torch.where(valid, (top + total.log())[:, 0], 0)
    p = torch.where(valid[:, None], e / total, 0)
    n = valid.sum()
    chosen = torch.where(valid[:, None], s["topk_idx"], E).long().flatten()
    counts = torch.zeros(E + 1, dtype=torch.int64, device="cuda").index_add_(0, chosen, torch.ones_like(chosen))
    counts[E] = n
    many = n.clamp(min=1).float()
    share, importance = counts[:E].float() * (E / c["k"]) / many, p.sum(0) / many
    losses = torch.stack(((share * importance).sum(), lse.square().sum() / many))
    a, b = _WEIGHTS
    dz = p * (share - (share * p).sum(1, keepdim=True)) * (a / many) + p * lse[:, None] * (2 * b / many)
    return {"losses": losses, "counts": counts.int(), "importance": importance, "lse": lse, "dlogits": s["add"] + dz if c["residual"] else dz}


def run(state):
    s, op = state, state["case"]["op"]
    if own:
        return _run_own(s)
    return {"norm": _plain_norm, "axes": _plain_axes, "balance": _plain_balance}[op](s)


def _run_own(s):
    from paper_2508_02317_amd import libmoe as L
    c = s["case"]
    if c["op"] == "norm":
        if c["back"]:
            dx, dw, db = L.moe_norm_bwd(s["dy"], s["x"], s["rstd"], s["mean"], s["weight"], add=s["residual"], out=s["out"], ws=s["ws"])
            return {"dx": dx, "dweight": dw, "dbias": db}
        y, h, mean, rstd = L.moe_norm_fwd(s["x"], s["weight"], s["bias"], eps=1e-6, rms=c["rms"], residual=s["residual"], out=s["out"])
        return {"h": h, "mean": mean, "rstd": rstd, "y": y}
    if c["op"] == "axes":
        if c["store"]:
            q = L.moe_kv_cache_write_axes(s["cache"], s["k"], s["v"], s["slots"], s["q"], s["positions"], s["cos"], s["sin"], s["pair_axis"], c["interleaved"],
                                          q_out=s["out"][0])
            return {"q": q, "k_cache": s["kc"], "v_cache": s["vc"]}
        turn = L.moe_rope_axes_bwd if c["back"] else L.moe_rope_axes_fwd
        q, k = turn(s["q"], s["k"], s["positions"], s["cos"], s["sin"], s["pair_axis"], c["interleaved"], out=s["out"])
        return {"q": q, "k": k}
    losses, counts, importance, lse = L.moe_balance_loss_fwd(s["logits"], s["topk_idx"], s["valid"], out=s["fwd"], ws=s["ws"])
    dlogits = L.moe_balance_loss_bwd(s["logits"], counts, lse, c["k"], *_WEIGHTS, valid=s["valid"], add=s["add"], out=s["dlogits"])
    return {"losses": losses, "counts": counts, "importance": importance, "lse": lse, "dlogits": dlogits}


# ---- the same in 64 bits ----------------------------------------------------------------------------------

def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "norm":
        return _exact_norm(c, s)
    if c["op"] == "axes":
        return _exact_axes(c, s)
    z, E = s["logits"].double(), c["experts"]
    keep = s["valid"].nonzero()[:, 0] if s["valid"] is not None else torch.arange(len(z), device="cuda")
    n, kept = max(len(keep), 1), z[keep]
    counts = torch.bincount(s["topk_idx"][keep].flatten().long(), minlength=E)
    p, lse = torch.softmax(kept, dim=1), torch.logsumexp(kept, dim=1)
    share = counts.double() * E / (c["k"] * n)
    losses = torch.stack((share @ p.mean(0), lse.square().mean())) if len(keep) else torch.zeros(2, dtype=torch.float64, device="cuda")
    a, b = _WEIGHTS
    dlogits, full = s["add"].double() if c["residual"] else torch.zeros_like(z), torch.zeros(len(z), dtype=torch.float64, device="cuda")
    dlogits[keep] += (a / n * (share - (p @ share)[:, None]) + 2 * b / n * lse[:, None]) * p
    full[keep] = lse
    return {"losses": losses, "counts": torch.cat((counts, torch.tensor([len(keep)], device="cuda"))).int(), "importance": p.sum(0) / n, "lse": full,
            "dlogits": dlogits}


def _exact_norm(c, s):
    """By the standard deviation and, for the gradients, by projections: dx is g without its parts along the centred row (and along ones)."""
    x, w = s["x"].double(), s["weight"].double()
    if not c["back"]:
        out = {}
        if c["residual"]:
            out["h"] = x + s["residual"].double()
            x = out["h"].to(s["x"].dtype).double()     # the norm is that of what is kept
        if not c["rms"]:
            out["mean"] = x.sum(-1) / c["dim"]
        var = (x * x).sum(-1) / c["dim"] if c["rms"] else x.var(-1, unbiased=False)
        out["rstd"] = (var + 1e-6) ** -0.5
        centred = x if c["rms"] else x - out["mean"][..., None]
        out["y"] = torch.einsum("...d,...,d->...d", centred, out["rstd"], w)
        if c["bias"]:
            out["y"] = out["y"] + s["bias"].double()
        return out
    centred = x if c["rms"] else x - x.mean(-1, keepdim=True)
    r = ((centred * centred).mean(-1, keepdim=True) + 1e-6) ** -0.5
    dy = s["dy"].double()
    g = dy * w
    along = (g * centred).sum(-1, keepdim=True) / c["dim"] * r * r
    dx = r * (g - along * centred)
    if not c["rms"]:
        dx = dx - r * g.mean(-1, keepdim=True)
    if c["residual"]:
        dx = dx + s["residual"].double()
    out = {"dx": dx, "dweight": (dy * (centred * r)).flatten(0, -2).sum(0)}
    if c["bias"]:
        out["dbias"] = dy.flatten(0, -2).sum(0)
    return out


def _exact_axes(c, s):
    """Each pair of elements as one complex number, times cos + i sin of its axis' position."""
    rot, axis = c["rot"], list(s["pair_axis"])
    half = rot // 2
    turn = torch.empty((c["tokens"], half), dtype=torch.complex128, device="cuda")
    for i in range(half):
        p = s["positions"][axis[i]].long()
        turn[:, i] = torch.complex(s["cos"][p, i].double(), s["sin"][p, i].double())
    if c["back"]:
        turn = turn.conj().resolve_conj()

    def turned(x):
        y, h = x.double(), x.shape[1]
        pairs = y[..., :rot].reshape(len(y), h, half, 2) if c["interleaved"] else y[..., :rot].reshape(len(y), h, 2, half).transpose(2, 3)
        z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn[:, None])
        y[..., :rot] = (z if c["interleaved"] else z.transpose(2, 3)).reshape(len(y), h, rot)
        return y

    if not c["store"]:
        return {n: turned(s[n]) for n in "qk"}
    out = {"q": turned(s["q"]), "k_cache": s["kc"].double(), "v_cache": s["vc"].double()}
    page, place = s["slots"] // _PAGE, s["slots"] % _PAGE
    out["k_cache"][page, :, place], out["v_cache"][page, :, place] = turned(s["k"]), s["v"].double()
    return out
