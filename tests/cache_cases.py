"""Plain 64-bit forms of the key/value cache's operators, from the layout and the formulas of include/squant.h alone."""
import functools
import math

import torch


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


@functools.lru_cache(maxsize=None)
def places(dim):
    """Byte offsets in a granule: code bytes and shifts of keys and values [16, dim], scales of keys and values [16, dim / 32]."""
    slabs = max(1, dim // 128)
    words, groups = dim // slabs // 8, dim // slabs // 32
    out = {n: torch.zeros((16, dim), dtype=torch.int64) for n in ("k", "v", "shift")}
    out |= {n: torch.zeros((16, dim // 32), dtype=torch.int64) for n in ("ks", "vs")}
    for t in range(16):
        for ch in range(dim):
            slab, word, e = ch // 8 // words, ch // 8 % words, ch % 8
            bit = 4 * (e // 2) + 16 * (e % 2)
            kw = (slab * 16 + t) * words + word % 4 * (words // 4) + word // 4
            vw = ((slab * 8 + t // 2) * 8 + word % 8) * 2 * (words // 8) + t % 2 * (words // 8) + word // 8
            out["k"][t, ch], out["v"][t, ch], out["shift"][t, ch] = 4 * kw + bit // 8, 8 * dim + 4 * vw + bit // 8, bit % 8
        for n in range(dim // 32):
            slab, r = divmod(n, groups)
            out["ks"][t, n] = 16 * dim + 2 * (t * (dim // 32) + n)
            out["vs"][t, n] = 17 * dim + 2 * (((slab * 8 + t // 2) * 2 + r % 2) * groups + r // 2 * 2 + t % 2)
    return out


def _scales(granules, at):
    low, high = granules[..., at].to(torch.int32), granules[..., at + 1].to(torch.int32)
    return ((high << 8 | low) << 16).view(torch.float32).double()


def parts(cache):
    """Codes of keys and values [pages, heads, page size, dim], and their scales [.., dim / 32], as doubles."""
    dim = cache.shape[3] // 18
    at = {n: t.to(cache.device) for n, t in places(dim).items()}
    got = []
    for n in ("k", "v"):
        c = cache[..., at[n]].to(torch.int32) >> at["shift"].to(torch.int32) & 15
        got.append((c - 16 * (c > 7)).double().flatten(2, 3))
        got.append(_scales(cache, at[n + "s"]).flatten(2, 3))
    return got[0], got[1], got[2], got[3]


def values(cache):
    """Keys and values [pages, heads, page size, dim] in fp64."""
    kc, ks, vc, vs = parts(cache)
    return kc * ks.repeat_interleave(32, -1), vc * vs.repeat_interleave(32, -1)


def scale_of(x):
    """Scales [.., dim / 32] in fp64 of values [.., dim]."""
    top = x.double().unflatten(-1, (-1, 32)).abs().amax(-1)
    step = top / torch.full_like(top, 7.0)
    unit = torch.ldexp(torch.ones_like(step), torch.frexp(step).exponent - 4)
    s = torch.round(step / unit) * unit
    s = torch.where(top < 2.0 ** -100, torch.zeros_like(s), s)
    return torch.where((top < 2.0 ** 120), s, torch.full_like(s, math.inf))


def stored(x):
    """What the cache makes of values [.., dim], in fp64."""
    s = scale_of(x).repeat_interleave(32, -1)
    plain = (s > 0) & (s < math.inf)
    code = torch.where(plain, torch.round(x.double() / torch.where(plain, s, torch.ones_like(s))), torch.zeros_like(s))
    return torch.where(s == math.inf, torch.full_like(s, math.nan), code * s)


class Batch:
    """Sequences of `lens` positions, `news` of them new, in pages in random order."""

    def __init__(self, lens, news, page_size, seed=0, spare=2, extra_rows=0):
        self.lens_list, self.news, self.page_size = list(lens), list(news), page_size
        width = max(1, -(-max(lens, default=0) // page_size))
        self.page_count = len(lens) * width + spare
        g = torch.Generator()
        g.manual_seed(seed)
        self.pages_list = torch.randperm(self.page_count, generator=g)[:len(lens) * width].view(len(lens), width)
        self.lens = torch.tensor(self.lens_list, dtype=torch.int32, device="cuda")
        self.pages = self.pages_list.to(torch.int32).cuda()
        self.starts = torch.tensor([0] + self.news, dtype=torch.int64).cumsum(0).to(torch.int32).cuda()
        self.rows = sum(self.news) + extra_rows
        self.args = (self.lens, self.pages, self.starts)

    def rows_of(self, b):
        first = sum(self.news[:b])
        return range(first, first + self.news[b])

    def sequence(self, full, b, n=None):
        """Positions 0 .. n of sequence b [n, heads, dim] out of [pages, heads, page size, dim]."""
        n = self.lens_list[b] if n is None else n
        return full[self.pages_list[b].to(full.device)].movedim(2, 1).flatten(0, 1)[:n]


def filled(batch, heads, dim, seed, dtype=torch.bfloat16, outliers=True):
    """A cache whose every position holds something, written by the plain form's own packing."""
    shape = (batch.page_count, heads, batch.page_size // 16, 16, dim)
    k = torch.randn(shape, generator=gen(seed), device="cuda")
    v = torch.randn(shape, generator=gen(seed + 1), device="cuda")
    if outliers:
        k = k * (1 + 3 * (torch.rand(dim, generator=gen(seed + 2), device="cuda") < 0.05))
    return pack(k.to(dtype), v.to(dtype))


def pack(k, v):
    """Cache [.., 18 dim] of keys and values [.., 16, dim]."""
    dim = k.shape[-1]
    at = {n: t.to(k.device) for n, t in places(dim).items()}
    out = torch.zeros((*k.shape[:-2], 18 * dim), dtype=torch.int32, device=k.device)
    for n, x in (("k", k), ("v", v)):
        s = scale_of(x)
        full = s.repeat_interleave(32, -1)
        plain = (full > 0) & (full < math.inf)
        code = torch.where(plain, torch.round(x.double() / torch.where(plain, full, torch.ones_like(full))), torch.zeros_like(full)).to(torch.int32) & 15
        flat = at[n].flatten()
        out.index_add_(-1, flat, (code << at["shift"].to(torch.int32)).flatten(-2))
        bits = s.float().view(torch.int32) >> 16 & 0xffff
        out[..., at[n + "s"].flatten()] = bits.flatten(-2) & 255
        out[..., at[n + "s"].flatten() + 1] = bits.flatten(-2) >> 8
    return out.to(torch.uint8)


def attention(q, batch, cache, scale=None):
    """Output and lse in fp64 of queries [rows, heads, dim]; rows in no sequence are None."""
    k_full, v_full = values(cache)
    rows, heads, dim = q.shape
    group = heads // cache.shape[1]
    scale = 1 / math.sqrt(dim) if scale is None else scale
    out = torch.zeros((rows, heads, dim), dtype=torch.float64, device="cuda")
    lse = torch.full((rows, heads), -math.inf, dtype=torch.float64, device="cuda")
    for b, n in enumerate(batch.lens_list):
        k, v = batch.sequence(k_full, b), batch.sequence(v_full, b)
        span = batch.rows_of(b)
        for i, row in enumerate(span):
            seen = n - len(span) + i + 1
            if seen <= 0:
                continue
            kk, vv = k[:seen].repeat_interleave(group, 1), v[:seen].repeat_interleave(group, 1)
            s = torch.einsum("hd,jhd->hj", q[row].double(), kk) * scale
            lse[row] = torch.logsumexp(s, -1)
            out[row] = torch.einsum("hj,jhd->hd", torch.softmax(s, -1), vv)
    return out, lse
