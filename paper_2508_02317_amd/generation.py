"""Generation beside the MoE layer: rotation tables, a paged key/value cache with its pages' book-keeping, and the attention half of a
transformer block over it.

    prompt   projection -> moe_kv_cache_write -> moe_kv_cache_read -> attention of the prompt's tokens (torch, in 32 bits) -> projection
    token    projection -> moe_kv_cache_write -> moe_paged_attn_decode -> projection

The projections are plain library products; rotation, cache and the attention of single tokens are calls into libmoe on the current
stream.  Which pages a sequence has is decided here, on the host, and reaches the device as four small tensors per step and layer, each
a copy that the host waits for.
"""
import math

import torch

from . import libmoe as L


def rope_frequencies(rot, base=10000.0, scaling="none", factor=1.0, original=None, low=1.0, high=32.0):
    """Angle per position of every pair, [rot / 2] float64 on the host: w_i = base ** (-2 i / rot), for a context `factor` times longer than
    the `original` one
      "linear"  all positions moved together: w_i / factor
      "base"    the base raised by factor ** (rot / (rot - 2)): the first pair keeps its w, the last one's falls by `factor`
      "parts"   pairs that turn more than `high` times over the original context keep their w, those that turn fewer than `low` times are
                moved together as by "linear", those between are mixed in proportion."""
    if rot % 2 or rot < 2:
        raise ValueError("rot must be a positive even number, got %r" % (rot,))
    if factor < 1.0:
        raise ValueError("factor must be at least 1, got %r" % (factor,))
    i = torch.arange(0, rot, 2, dtype=torch.float64)
    if scaling == "base":
        if rot < 4:
            raise ValueError("a raised base needs two pairs or more")
        return (base * factor ** (rot / (rot - 2))) ** (-i / rot)
    w = base ** (-i / rot)
    if scaling == "none":
        return w
    if scaling == "linear":
        return w / factor
    if scaling == "parts":
        if original is None or not high > low:
            raise ValueError('"parts" needs the original context and high > low')
        keep = ((original * w / (2 * math.pi) - low) / (high - low)).clamp(0.0, 1.0)
        return w * (keep + (1.0 - keep) / factor)
    raise ValueError("unknown scaling %r" % (scaling,))


def rope_amplitude(factor):
    """Amplitude that goes with "parts": scores of a context `factor` times longer are sharpened by its square."""
    return 1.0 if factor <= 1.0 else 0.1 * math.log(factor) + 1.0


class PagedKVCache:
    """Keys and values of one attention layer in pages of page_size tokens, and the pages of every sequence.

    eight_bit: E4M3 codes with a power-of-two scale per 32 elements instead of bfloat16 (33/64 of the memory and of what attention reads)."""

    def __init__(self, pages, page_size, heads, dim, dtype=torch.bfloat16, eight_bit=False, device="cuda"):
        if eight_bit and dtype is not torch.bfloat16:
            raise ValueError("an 8-bit cache goes with bfloat16 activations")
        shape = (pages, heads, page_size, dim)
        mk = lambda n, t: torch.zeros(shape[:3] + (n,), dtype=t, device=device)
        if eight_bit:
            self.k, self.v, self.k_scales, self.v_scales = (mk(n, torch.uint8) for n in (dim, dim, dim // 32, dim // 32))
        else:
            self.k, self.v, self.k_scales, self.v_scales = mk(dim, dtype), mk(dim, dtype), None, None
        self.view = L.moe_kv_cache(self.k, self.v, self.k_scales, self.v_scales)
        self.page_size, self.device = page_size, torch.device(device)
        self.free = list(range(pages - 1, -1, -1))
        self.pages_of, self.length = {}, {}

    def open(self, seq):
        if seq in self.length:
            raise ValueError("sequence %r is open" % (seq,))
        self.pages_of[seq], self.length[seq] = [], 0

    def close(self, seq):
        self.free.extend(reversed(self.pages_of.pop(seq)))
        del self.length[seq]

    def grow(self, seqs, counts):
        """Places for counts[i] new tokens of seqs[i] -> slots [sum] i64, positions [sum] i32, pages [B, widest] i32, lens [B] i32, all on
        the device.  Nothing changes where the arguments do not fit (ValueError) or the free pages do not suffice (MemoryError)."""
        if len(set(seqs)) != len(seqs):
            raise ValueError("a sequence is named twice")
        if len(counts) != len(seqs) or min(counts, default=0) < 0:
            raise ValueError("every sequence needs a number of new tokens of 0 or more")
        ps = self.page_size
        need = [-(-(self.length[s] + n) // ps) - len(self.pages_of[s]) for s, n in zip(seqs, counts)]
        if sum(need) > len(self.free):
            raise MemoryError("%d pages wanted, %d free" % (sum(need), len(self.free)))
        slots, positions = [], []
        for s, n, new in zip(seqs, counts, need):
            mine, at = self.pages_of[s], self.length[s]
            mine.extend(self.free.pop() for _ in range(new))
            positions.extend(range(at, at + n))
            slots.extend(mine[t // ps] * ps + t % ps for t in range(at, at + n))
            self.length[s] = at + n
        widest = max([len(self.pages_of[s]) for s in seqs] + [1])
        table = [p for s in seqs for p in self.pages_of[s] + [0] * (widest - len(self.pages_of[s]))]
        lens = [self.length[s] for s in seqs]
        to = lambda v, t: torch.tensor(v, dtype=t).to(self.device)
        try:
            return to(slots, torch.int64), to(positions, torch.int32), to(table, torch.int32).view(len(seqs), widest), to(lens, torch.int32)
        except BaseException:                          # no memory on the device
            self.shrink(seqs, counts)
            raise

    def shrink(self, seqs, counts):
        """Takes the last counts[i] tokens of seqs[i] back, and the pages that held nothing else: after a grow of the same arguments everything, the
        order of the free pages included, is as it was before.  Nothing changes where the arguments do not fit (ValueError)."""
        if len(set(seqs)) != len(seqs) or len(counts) != len(seqs) or not all(0 <= n <= self.length[s] for s, n in zip(seqs, counts)):
            raise ValueError("every sequence needs a number of tokens that it has")
        for s, n in zip(reversed(seqs), reversed(counts)):
            self.length[s] -= n
            while len(self.pages_of[s]) > -(-self.length[s] // self.page_size):
                self.free.append(self.pages_of[s].pop())


class CachedAttention:
    """The attention half of a block: y = W_out attention(rope(q), rope(k), v) with [q | k | v] = x W_qkv^T, the keys and values of earlier tokens in a
    PagedKVCache.  w_qkv [(heads + 2 kv_heads) dim, d], w_out [d, heads dim]; cos, sin [n_pos, rot / 2] f32 (moe_rope_table)."""

    def __init__(self, cache, heads, w_qkv, w_out, cos, sin, interleaved=False, window=0):
        self.cache, self.heads, self.kv_heads, self.dim = cache, heads, cache.view.heads, cache.view.dim
        self.w_qkv, self.w_out, self.cos, self.sin, self.interleaved, self.window = w_qkv, w_out, cos, sin, interleaved, window
        if w_qkv.shape[0] != (heads + 2 * self.kv_heads) * self.dim or w_out.shape[1] != heads * self.dim:
            raise ValueError("w_qkv must have (heads + 2 kv_heads) dim rows and w_out heads dim columns")

    def _step(self, x, seqs, counts, attend):
        """Projections around attend(q, pages, lens) -> [T, heads, dim] with the rows of x stored: q their rotated queries [T, heads, dim], a view of the
        projection's output, pages and lens those of the sequences.  What does not fit is refused before a sequence has grown, and where anything
        raises after that (memory that runs out, a call that refuses), the growth is taken back: no sequence keeps places that were not written."""
        d = self.w_qkv.shape[1]
        if x.dim() != 2 or x.shape[1] != d or len(x) != sum(counts):
            raise ValueError("rows of %d elements for %d new tokens are wanted, got %s" % (d, sum(counts), tuple(x.shape)))
        if x.dtype is not self.w_qkv.dtype or x.device != self.w_qkv.device:
            raise TypeError("rows must be %s on %s like the weights, got %s on %s" % (self.w_qkv.dtype, self.w_qkv.device, x.dtype, x.device))
        if max((self.cache.length[s] + n for s, n in zip(seqs, counts)), default=0) > self.cos.shape[0]:
            raise ValueError("the rotation table ends at position %d" % self.cos.shape[0])
        slots, positions, pages, lens = self.cache.grow(seqs, counts)
        try:
            qkv = torch.mm(x, self.w_qkv.t()).view(len(x), self.heads + 2 * self.kv_heads, self.dim)
            q, k, v = qkv.split([self.heads, self.kv_heads, self.kv_heads], dim=1)
            q = L.moe_kv_cache_write(self.cache.view, k, v, slots, q, positions, self.cos, self.sin, self.interleaved, q_out=q)
            return torch.mm(attend(q, pages, lens).view(len(x), self.heads * self.dim), self.w_out.t())
        except BaseException:
            self.cache.shrink(seqs, counts)
            raise

    def token(self, x, seqs):
        """One new token x[i] of every sequence seqs[i] -> [B, d]."""
        return self._step(x, seqs, [1] * len(seqs), lambda q, pages, lens: L.moe_paged_attn_decode(q, self.cache.view, pages, lens, window=self.window)[0])

    def prompt(self, x, seqs, counts):
        """counts[i] new tokens of seqs[i], their rows of x one sequence after the other -> [sum(counts), d].  Every token attends to what its
        sequence has in the cache up to itself."""
        return self._step(x, seqs, counts, lambda q, pages, lens: self._attend_prompt(q, pages, counts, [self.cache.length[s] for s in seqs]))

    def _attend_prompt(self, q, pages, counts, ends):
        starts = torch.tensor([0] + ends, dtype=torch.int32).cumsum(0, dtype=torch.int32).to(q.device)
        k, v = L.moe_kv_cache_read(self.cache.view, pages, starts, rows=sum(ends))
        y, row, key = torch.empty_like(q, memory_format=torch.contiguous_format), 0, 0
        for n, end in zip(counts, ends):
            g = self.heads // self.kv_heads
            kk, vv = (t[key:key + end].float().repeat_interleave(g, dim=1).transpose(0, 1).contiguous() for t in (k, v))
            score = (q[row:row + n].float().transpose(0, 1).contiguous() @ kk.transpose(1, 2).contiguous()) * self.dim ** -0.5
            t = torch.arange(end, device=q.device)
            own = t[end - n:, None]
            hidden = (t > own) | (t <= own - self.window) if self.window else t > own
            y[row:row + n] = (score.masked_fill(hidden, -math.inf).softmax(-1) @ vv).transpose(0, 1).to(y.dtype)
            row, key = row + n, key + end
        return y
