"""Workloads of the attention side of a serving and training step: rotary positions, the paged key/value cache, and the attention of
one new token over it.

A case is a dict of sizes and options.  `prepare` makes what a program holds before the call (projected queries, keys and values, the
rotation table, a cache with its page table), `run` is one pass, `exact` the same in 64 bits, `work` the bytes and operations a pass
cannot do without.  With `own` false `run` uses elementary torch operations in 32 bits; with `own` true the library's entry points.

Kinds (`op`):
  rope    queries and keys of a training micro-batch rotated by their positions, or the gradients rotated back (`back`)
  write   the same rotation at prefill, with keys and values stored into the pages of a cache
  append  a chunk is rotated and stored in 8 bits, and the whole contexts are read back for the chunk's attention
  read    cached keys and values of several sequences gathered from their pages into packed rows
  token   one generation step: the new token of every sequence is rotated and stored, then attends to its context
  attend  the attention of one new token per sequence alone

The cache is [pages, kv_heads, page, dim] for keys and the same for values, in float32, bfloat16, or 8 bits (E4M3 codes with one
power-of-two scale per 32 elements of `dim`, scales [pages, kv_heads, page, dim / 32], value = 2^(scale - 127) * code).
"""
import math

import torch

own = False

_DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
_BASE = 1e6                                            # base of the rotation's frequencies
_TOP_BYTES = 1.2e9                                     # of the largest listed case, about


def _case(op, **options):
    c = dict(op=op, heads=32, kv_heads=4, dim=128, rot=128, interleaved=False, dtype="bf16", tokens=0, back=False, fused=False,
             seqs=0, longest=0, ragged=True, page=16, cache="bf16", window=0, positions=0)
    c.update(options)
    return c


def listed():
    cases = {
        # a full-precision parity run: few tokens, a head per key head
        "rope_256_f32": _case("rope", tokens=256, heads=8, kv_heads=8, dim=64, rot=64, dtype="f32"),
        # one 8K-token micro-batch, queries and keys being views of one projection's output
        "rope_8k": _case("rope", tokens=8192, fused=True),
        # gradients of one sequence shard of a 160K-token sequence
        "rope_40k_back": _case("rope", tokens=40960, back=True, positions=122880),
        # gradients of an odd last micro-batch, neighbouring pairs, half of each head rotated
        "rope_odd_partial_back": _case("rope", tokens=1531, heads=16, kv_heads=2, rot=64, interleaved=True, back=True),
        # prefill of 8K tokens of several prompts
        "write_8k": _case("write", tokens=8192, seqs=6, longest=4096, page=64, fused=True),
        # chunked prefill over an 8-bit cache: an odd chunk goes in, 8 contexts come back
        "append_2k_mx8": _case("append", tokens=2047, seqs=8, longest=8192, page=64, cache="mx8"),
        # contexts of a batch copied out of their pages, as for a move to another device or a prompt shared by later requests
        "read_40k": _case("read", seqs=12, longest=8192, page=16),
        # one generation step of a small batch
        "token_16": _case("token", seqs=16, longest=4096, page=16, fused=True),
        # one conversation alone: latency
        "attend_1_2k": _case("attend", seqs=1, longest=2047, ragged=False, page=16),
        # a full-precision parity run: few heads, sliding window
        "attend_4_f32_window": _case("attend", seqs=4, longest=700, heads=8, kv_heads=8, dim=64, rot=64, dtype="f32", cache="f32", window=256),
        # a busy server: sequences of very different lengths, an empty place and a first token among them
        "attend_64": _case("attend", seqs=64, longest=8192, page=64),
        # long contexts in 8 bits
        "attend_32_40k_mx8": _case("attend", seqs=32, longest=40960, page=128, cache="mx8"),
    }
    return [dict(c, name=n) for n, c in cases.items()]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rope", "rope", "write", "append", "read", "token", "attend", "attend", "attend"])
    dim = rng.choice([64, 128, 128, 192, 256])
    kv_heads = rng.choice([1, 2, 4, 8])
    heads = kv_heads * rng.choice([1, 2, 4, 7, 8, 12, 16])
    dtype = "f32" if rng.random() < 0.15 else "bf16"
    cache = dtype if dtype == "f32" else rng.choice(["bf16", "mx8"])
    if op == "append":
        dtype, cache = "bf16", "mx8"
    if op in ("write", "token"):                       # they return the cache, which stands for itself in these types
        cache = dtype
    c = _case(op, dim=dim, kv_heads=kv_heads, heads=heads, dtype=dtype, cache=cache, rot=rng.choice([dim, dim, dim // 2]),
              interleaved=rng.random() < 0.4, page=rng.choice([16, 32, 64, 128]))
    if op in ("rope", "write", "token"):
        c["fused"] = rng.random() < 0.5
    if op == "rope":
        c.update(tokens=_log_int(rng, 1, 40960), back=rng.random() < 0.5, positions=rng.choice([0, 0, 30000, 122880]))
    elif op in ("write", "append"):
        c.update(tokens=_log_int(rng, 16, 8192), seqs=rng.randint(1, 16), longest=_log_int(rng, 64, 16384))
        c["longest"] = max(c["longest"], c["tokens"])  # a sequence of at least its share of the new tokens
    else:
        c.update(seqs=_log_int(rng, 1, 128), longest=_log_int(rng, 1, 40960), ragged=rng.random() < 0.7)
    if op in ("token", "attend"):
        c["window"] = rng.choice([0, 0, 0, 128, 1000])
    # no more memory moved, and no more cache held, than in the largest listed cases
    while work(c)["bytes"] > 0.8 * _TOP_BYTES or _cache_bytes(c) > _TOP_BYTES:
        if c["seqs"] > 1:
            c["seqs"] = (c["seqs"] + 1) // 2
        elif c["op"] in ("rope", "write", "append"):
            c["tokens"] = (c["tokens"] + 1) // 2
            c["longest"] = max((c["longest"] + 1) // 2, c["tokens"]) if c["longest"] else 0
        else:
            c["longest"] = (c["longest"] + 1) // 2
    return c


# ---- sizes that follow from a case alone ------------------------------------------------------------------

def _lens(c):
    """Context lengths, the new tokens included: the longest, and where ragged an empty place (attend, read), a first token and a spread."""
    n, top = c["seqs"], c["longest"]
    if not c["ragged"]:
        return [top] * n
    lens = [max(1, int(top * math.fmod(0.618034 * i + 1e-9, 1.0))) if i else top for i in range(n)]
    if n >= 8:
        lens[2], lens[5] = 1, 0 if c["op"] in ("attend", "read") else 1
    if c["op"] in ("write", "append"):
        new = _new_tokens(c)
        lens = [max(a, b) for a, b in zip(lens, new)]
    return lens


def _new_tokens(c):
    """New tokens of every sequence: one each, or the chunk dealt out unevenly."""
    n = c["seqs"]
    if c["op"] == "token":
        return [1] * n
    cuts = [int(c["tokens"] * (i / n) ** 1.3) for i in range(n)] + [c["tokens"]]
    return [b - a for a, b in zip(cuts, cuts[1:])]


def _row_bytes(c):
    """Of keys and values of one token of one head in the cache."""
    d = c["dim"]
    return 2 * {"f32": 4 * d, "bf16": 2 * d, "mx8": d + d // 32}[c["cache"]]


def _cache_bytes(c):
    return sum(-(-n // c["page"]) * c["page"] for n in _lens(c)) * c["kv_heads"] * _row_bytes(c) if c["seqs"] else 0


def work(case):
    c = case
    d, es = c["dim"], 4 if c["dtype"] == "f32" else 2
    table = c["rot"] * 4                               # cosines and sines of a position
    q, kv = c["heads"] * d * es, c["kv_heads"] * d * es
    if c["op"] == "rope":
        return {"bytes": c["tokens"] * (2 * (q + kv) + table + 4), "flops": c["tokens"] * 3 * c["rot"] * (c["heads"] + c["kv_heads"])}
    lens = _lens(c)
    row, pages = c["kv_heads"] * _row_bytes(c), sum(-(-n // c["page"]) for n in lens) * 4
    if c["op"] == "read":
        return {"bytes": sum(lens) * (row + 2 * kv) + pages, "flops": sum(lens) * 2 * c["kv_heads"] * d}
    new = sum(_new_tokens(c)) if c["op"] != "attend" else 0
    store = new * (2 * q + 2 * kv + row + table + 12)
    turn = new * 3 * c["rot"] * (c["heads"] + c["kv_heads"])
    if c["op"] == "write":
        return {"bytes": store, "flops": turn}
    if c["op"] == "append":
        return {"bytes": store + sum(lens) * (row + 2 * kv) + pages, "flops": turn + sum(lens) * 2 * c["kv_heads"] * d}
    seen = sum(min(n, c["window"]) if c["window"] else n for n in lens)
    attend = {"bytes": seen * row + pages + c["seqs"] * (2 * q + 4 * c["heads"]), "flops": seen * c["heads"] * 4 * d}
    return {k: attend[k] + (store, turn)[k == "flops"] for k in attend} if c["op"] == "token" else attend


# ---- inputs -----------------------------------------------------------------------------------------------

def _normal(gen, shape, std, dtype):
    """N(0, std) rounded to dtype, drawn slab by slab so that no fp32 copy of a large cache exists."""
    out = torch.empty(shape, dtype=dtype, device="cuda")
    flat, step = out.view(-1), 1 << 26
    for s in range(0, flat.numel(), step):
        part = flat[s:s + step]
        part.copy_(torch.randn(part.numel(), generator=gen, device="cuda").mul_(std))
    return out


def _table(n_pos, rot):
    """Cosines and sines [n_pos, rot / 2] of the angles, formed in 64 bits and rounded once."""
    w = _BASE ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)
    a = torch.arange(n_pos, dtype=torch.float64, device="cuda")[:, None] * w
    return a.cos().float(), a.sin().float()


def _heads(gen, c, rows, groups):
    """[rows, h, dim] for each h of `groups`: tensors of their own, or views of one projection's output."""
    d, dtype = c["dim"], _DTYPE[c["dtype"]]
    if not c["fused"]:
        return [_normal(gen, (rows, h, d), 1.0, dtype) for h in groups]
    whole = _normal(gen, (rows, sum(groups), d), 1.0, dtype)
    return list(whole.split(groups, dim=1))


def _sharpness(gen, c):
    """Scale of each head's queries: some look broadly, some at few tokens."""
    return 0.5 + 3.0 * torch.rand((c["heads"], 1), generator=gen, device="cuda")


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    s = {"case": c}
    dtype, d, kvh = _DTYPE[c["dtype"]], c["dim"], c["kv_heads"]
    if c["op"] == "rope":
        T = c["tokens"]
        s["q"], s["k"] = _heads(gen, c, T, [c["heads"], kvh])
        s["cos"], s["sin"] = _table(c["positions"] + T, c["rot"])
        s["positions"] = torch.arange(c["positions"], c["positions"] + T, dtype=torch.int32, device="cuda")
        if own:
            s["out"] = (torch.empty((T, c["heads"], d), dtype=dtype, device="cuda"), torch.empty((T, kvh, d), dtype=dtype, device="cuda"))
        return s
    # a cache in use: the sequences' pages lie anywhere in it, and the sequences in any order
    order = torch.randperm(c["seqs"], generator=gen, device="cuda").tolist()
    lens = [_lens(c)[i] for i in order]
    page = c["page"]
    pages = [-(-n // page) for n in lens]
    n_pages, widest = sum(pages) + 3, max(max(pages), 1)
    table = torch.zeros((c["seqs"], widest), dtype=torch.int32)
    free = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32).cpu()
    at = 0
    for b, n in enumerate(pages):
        table[b, :n] = free[at:at + n]
        at += n
    s["pages"], s["longest"] = table.cuda(), max(lens)
    s["lens"] = torch.tensor(lens, dtype=torch.int32).cuda()
    shape = (n_pages, kvh, page, d)
    if c["cache"] == "mx8":
        codes = lambda: _codes(_normal(gen, shape, 1.0, torch.bfloat16))
        (s["kc"], s["ks"]), (s["vc"], s["vs"]) = codes(), codes()
    else:
        s["kc"], s["vc"] = (_normal(gen, shape, 1.0, dtype) for _ in range(2))
        s["ks"] = s["vs"] = None
    if c["op"] in ("read", "append"):
        starts = [0]
        for n in lens:
            starts.append(starts[-1] + n)
        s["rows"] = starts[-1]
        s["row_start"] = torch.tensor(starts, dtype=torch.int32).cuda()
    if c["op"] in ("write", "append", "token"):
        new = s["new"] = [_new_tokens(c)[i] for i in order]
        seq = torch.repeat_interleave(torch.arange(c["seqs"]), torch.tensor(new))
        pos = torch.cat([torch.arange(n - m, n) for n, m in zip(lens, new)])
        s["slots"] = (table[seq, pos // page].long() * page + pos % page).cuda()
        s["positions"] = pos.to(torch.int32).cuda()
        s["q"], s["k"], s["v"] = _heads(gen, c, len(seq), [c["heads"], kvh, kvh])
        s["cos"], s["sin"] = _table(max(lens), c["rot"])
    elif c["op"] == "attend":
        s["q"] = (_normal(gen, (c["seqs"], c["heads"], d), 1.0, torch.float32) * _sharpness(gen, c)).to(dtype)
    if own:
        from paper_2508_02317_amd import libmoe as L
        s["cache"] = L.moe_kv_cache(s["kc"], s["vc"], s["ks"], s["vs"])
        if "k" in s:
            s["q_out"] = torch.empty(s["q"].shape, dtype=dtype, device="cuda")
        if "rows" in s:
            s["out"] = tuple(torch.empty((s["rows"], kvh, d), dtype=dtype, device="cuda") for _ in range(2))
        if c["op"] in ("token", "attend"):
            s["out"], s["lse"] = torch.empty(s["q"].shape, dtype=dtype, device="cuda"), torch.empty(s["q"].shape[:2], device="cuda")
            n = L.lib.moe_paged_attn_decode_workspace_bytes(c["seqs"], c["heads"], kvh, d, page, widest)
            s["ws"] = torch.empty(n, dtype=torch.uint8, device="cuda")
    return s


# ---- the plain forms --------------------------------------------------------------------------------------

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


def _by_power(v, e):
    """v 2^e for whole e from -254 to 254, exact where the result has a place in 32 bits: the factors are made of their bits."""
    half = e // 2
    return v * ((half + 127).int() << 23).view(torch.float32) * ((e - half + 127).int() << 23).view(torch.float32)


def _codes(x):
    """Values [..., d] -> E4M3 codes and scale codes [..., d / 32], both uint8."""
    v = x.float().unflatten(-1, (-1, 32))
    _, e = torch.frexp(v.abs().amax(-1))               # amax = m 2^e, 1/2 <= m < 1
    scale = (e - 9 + 127).clamp(0, 254)
    scale = torch.where(v.abs().amax(-1) > 0, scale, 0)
    q = _by_power(v, 127 - scale[..., None]).clamp(-448, 448).to(torch.float8_e4m3fn)
    return q.view(torch.uint8).flatten(-2), scale.to(torch.uint8)


def _values(codes, scales):
    v = codes.view(torch.float8_e4m3fn).float().unflatten(-1, (-1, 32))
    return _by_power(v, scales.int()[..., None] - 127).flatten(-2)


def _fetch(s, which, page, at):
    """Cached rows [..., kv_heads, d] in 32 bits at (page, at) of the same leading shape."""
    rows = s[which + "c"][page, :, at]
    return rows.float() if s[which + "s"] is None else _values(rows, s[which + "s"][page, :, at])


def _plain_store(s):
    c = s["case"]
    cos, sin = s["cos"][s["positions"].long()], s["sin"][s["positions"].long()]
    page, at = s["slots"] // c["page"], s["slots"] % c["page"]
    k = _turn(s["k"], cos, sin, c["interleaved"])
    if c["cache"] == "mx8":
        s["kc"][page, :, at], s["ks"][page, :, at] = _codes(k)
        s["vc"][page, :, at], s["vs"][page, :, at] = _codes(s["v"])
    else:
        s["kc"][page, :, at], s["vc"][page, :, at] = k.to(s["kc"].dtype), s["v"].to(s["vc"].dtype)
    return _turn(s["q"], cos, sin, c["interleaved"]).to(s["q"].dtype)


def _plain_read(s):
    c = s["case"]
    row = torch.arange(s["rows"], device="cuda", dtype=torch.int32)
    b = torch.searchsorted(s["row_start"], row, right=True) - 1
    t = row - s["row_start"][b]
    page, at = s["pages"][b, t // c["page"]].long(), t.long() % c["page"]
    return tuple(_fetch(s, w, page, at).to(_DTYPE[c["dtype"]]) for w in "kv")


def _plain_attend(s, q):
    c = s["case"]
    B, h, d = q.shape
    g = h // c["kv_heads"]
    t = torch.arange(s["longest"], device="cuda")
    page = s["pages"][:, t // c["page"]].long()
    n = s["lens"][:, None]
    seen = (t < n) & (t >= n - c["window"]) if c["window"] else t < n
    k = _fetch(s, "k", page, t % c["page"]).transpose(1, 2)                  # [B, kv_heads, L, d]
    score = q.float().view(B, -1, g, d) @ k.transpose(2, 3).contiguous() / math.sqrt(d)
    del k
    seen = seen[:, None, None]
    score = torch.where(seen, score, -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.where(seen, (score - torch.where(top > -math.inf, top, 0)).exp(), 0)
    total = p.sum(-1, keepdim=True)
    v = torch.where(seen[:, 0, 0, :, None, None], _fetch(s, "v", page, t % c["page"]), 0).transpose(1, 2)
    out = (p / torch.where(total > 0, total, 1)) @ v.contiguous()
    return {"out": out.reshape(B, h, d).to(q.dtype), "lse": (top + total.log()).reshape(B, h)}


def run(state):
    s, c = state, state["case"]
    if own:
        return _run_own(s)
    if c["op"] == "rope":
        cos, sin = s["cos"][s["positions"].long()], s["sin"][s["positions"].long()]
        sin = -sin if c["back"] else sin
        return {n: _turn(s[n], cos, sin, c["interleaved"]).to(s[n].dtype) for n in "qk"}
    out = {}
    if c["op"] in ("write", "append", "token"):
        out["q"] = _plain_store(s)
    if c["op"] in ("write", "token"):
        out.update(k_cache=s["kc"], v_cache=s["vc"])
    if c["op"] in ("read", "append"):
        out["k"], out["v"] = _plain_read(s)
    if c["op"] in ("token", "attend"):
        out.update(_plain_attend(s, out.get("q", s["q"])))
    return out


def _run_own(s):
    from paper_2508_02317_amd import libmoe as L
    c = s["case"]
    if c["op"] == "rope":
        turn = L.moe_rope_bwd if c["back"] else L.moe_rope_fwd
        q, k = turn(s["q"], s["k"], s["positions"], s["cos"], s["sin"], c["interleaved"], out=s["out"])
        return {"q": q, "k": k}
    out = {}
    if c["op"] in ("write", "append", "token"):
        out["q"] = L.moe_kv_cache_write(s["cache"], s["k"], s["v"], s["slots"], s["q"], s["positions"], s["cos"], s["sin"], c["interleaved"],
                                        q_out=s["q_out"])
    if c["op"] in ("write", "token"):
        out.update(k_cache=s["kc"], v_cache=s["vc"])
    if c["op"] in ("read", "append"):
        out["k"], out["v"] = L.moe_kv_cache_read(s["cache"], s["pages"], s["row_start"], out=s["out"])
    if c["op"] in ("token", "attend"):
        out["out"], out["lse"] = L.moe_paged_attn_decode(out.get("q", s["q"]), s["cache"], s["pages"], s["lens"], window=c["window"], out=s["out"],
                                                         lse=s["lse"], ws=s["ws"])
    return out


# ---- the same in 64 bits ----------------------------------------------------------------------------------

def _exact_turn(x, cos, sin, interleaved):
    """Each pair of elements as one complex number, times cos + i sin."""
    rot, h = 2 * cos.shape[1], x.shape[1]
    y = x.double()
    pairs = y[..., :rot].reshape(len(y), h, -1, 2) if interleaved else y[..., :rot].reshape(len(y), h, 2, -1).transpose(2, 3)
    z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * torch.complex(cos.double(), sin.double())[:, None])
    y[..., :rot] = (z if interleaved else z.transpose(2, 3)).reshape(len(y), h, rot)
    return y


def _two_to(e):
    """2^e in 64 bits for whole e, made of its bits (a library's power may be off in the last one, which a tie would show)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_block_scaled(x):
    """What values [..., d] become in 8 bits: three mantissa bits below the leading one, down to 2^-6 of a scale 2^(floor(log2 top) - 8)."""
    v = x.double().unflatten(-1, (-1, 32))
    top = v.abs().amax(-1, keepdim=True)
    scale = _two_to((torch.frexp(torch.where(top > 0, top, 1.0)).exponent - 9).clamp(min=-127))
    step = _two_to((torch.frexp(v / scale).exponent - 1).clamp(min=-6) - 3)
    return ((v / scale / step).round() * step).clamp(-448, 448).mul(scale).flatten(-2)


def exact(case, seed):
    c, s = case, prepare(case, seed)
    out = {}
    if c["op"] == "rope":
        cos, sin = (s[n][s["positions"].long()] for n in ("cos", "sin"))
        return {n: _exact_turn(s[n], cos, -sin if c["back"] else sin, c["interleaved"]) for n in "qk"}
    page = c["page"]

    def cached(which, b, n):
        """[n, kv_heads, d] of a sequence's context as the prepared cache holds it."""
        t = torch.arange(n, device="cuda")
        p, at = s["pages"][b, t // page].long(), t % page
        rows = s[which + "c"][p, :, at]
        if c["cache"] != "mx8":
            return rows.double()
        return (rows.view(torch.float8_e4m3fn).double().unflatten(-1, (-1, 32)) * _two_to(s[which + "s"][p, :, at].long()[..., None] - 127)).flatten(-2)

    lens = s["lens"].tolist()
    held = lambda x, as_type: x.to(as_type).double()                         # what a cache of that type keeps
    new = {}
    if c["op"] in ("write", "append", "token"):
        cos, sin = (s[n][s["positions"].long()] for n in ("cos", "sin"))
        out["q"] = _exact_turn(s["q"], cos, sin, c["interleaved"])
        new = {"k": _exact_turn(s["k"], cos, sin, c["interleaved"]), "v": s["v"].double()}
        if c["cache"] == "mx8":
            new = {n: _exact_block_scaled(x) for n, x in new.items()}
    if c["op"] in ("write", "token"):
        for n in "kv":
            full = s[n + "c"].double()
            full[s["slots"] // page, :, s["slots"] % page] = new[n]
            out[n + "_cache"] = full
    if c["op"] in ("read", "append"):
        for n in "kv":
            parts, taken = [], 0
            for b, length in enumerate(lens):
                rows = cached(n, b, length)
                if new:                                                       # a sequence's new tokens end its context
                    m = s["new"][b]
                    rows[length - m:] = new[n][taken:taken + m]
                    taken += m
                parts.append(rows)
            out[n] = torch.cat(parts)
    if c["op"] in ("token", "attend"):
        q = out["q"].to(s["q"].dtype).double() if "q" in out else s["q"].double()
        g, y, lse = c["heads"] // c["kv_heads"], [], []
        for b, length in enumerate(lens):
            k, v = cached("k", b, length), cached("v", b, length)
            if new:
                k[length - 1], v[length - 1] = held(new["k"][b], s["kc"].dtype), held(new["v"][b], s["vc"].dtype)
            if c["window"]:
                k, v = k[-c["window"]:], v[-c["window"]:]
            k, v = (x.transpose(0, 1).repeat_interleave(g, dim=0) for x in (k, v))
            score = (k @ q[b][:, :, None])[..., 0] * c["dim"] ** -0.5          # [heads, L]
            lse.append(torch.logsumexp(score, dim=1))
            y.append((torch.softmax(score, dim=1)[:, None] @ v)[:, 0])
        out["out"], out["lse"] = torch.stack(y), torch.stack(lse)
    return out
