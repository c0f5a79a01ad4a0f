"""The calls that the operators of a key/value cache held in 4 bits are measured by.

A cache is a uint8 tensor [pages, kv heads, page size / 16, 18 * head dim]: for each page and head, granules of 16 tokens.  32
neighbouring channels of a token's key or value share a scale, absmax / 7 rounded to four significant bits; the codes are
rint(x / scale), in -7..7.  A granule holds the codes of its keys, of its values, then the scales (bfloat16) of both.  Rows
starts[b] .. starts[b + 1] of k, v, q and the outputs are the last positions of sequence b, which has lens[b] tokens in all;
position p lies in page pages[b][p // page size].  Three operators:

  "write"      new tokens' keys and values into the cache, and what it then stands for
  "read"       keys and values of whole sequences as 16-bit floats
  "attention"  softmax attention of each sequence's newest tokens over all of its tokens, causal; query head h reads kv head
               h // group

Head counts and dimensions are those of common grouped-query layers of 4096 and 8192 features, and odd ones; sequences have
from one token to 131,072.

Fields of a case:
  op                       one of the above
  dtype                    "bf16" or "fp16" (k, v, q and the outputs)
  heads, group, dim, page  kv heads, query heads of each, head dimension, tokens of a page
  batch, shortest, longest sequences and their tokens (spread over the logarithm; the first has the longest)
  few, many                new tokens of a sequence (at most what it has; 0: all of them)
  lse                      the logarithms of the softmax sums are asked for too
"""
import math
import random

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
_CASE = {"dtype": "bf16", "heads": 8, "group": 4, "dim": 128, "page": 64, "batch": 1, "few": 1, "many": 1, "lse": False}


def _case(op, name=None, **kw):
    c = dict(_CASE, op=op, **kw)
    return dict(c, name=name) if name else c


def listed():
    return [
        # a decoding step's keys and values: one token of each sequence
        _case("write", "write_step", batch=48, shortest=20, longest=4000),
        # a batch of prompts, packed
        _case("write", "write_prompts", batch=6, shortest=300, longest=8000, few=0, many=0),
        # a short sequence of an odd length, to be handed on
        _case("read", "read_short", dtype="fp16", heads=5, dim=64, page=16, shortest=333, longest=333, few=0, many=0),
        # a batch's caches back to 16 bits, to move them to another format
        _case("read", "read_batch", batch=9, shortest=500, longest=16000, page=128, few=0, many=0),
        # one sequence's next token: latency
        _case("attention", "step_one", shortest=777, longest=777),
        # a batch of sequences of different lengths, one token each
        _case("attention", "step_batch", batch=64, shortest=200, longest=8192),
        # one very long sequence
        _case("attention", "step_long", group=8, shortest=131072, longest=131072, lse=True),
        # wide heads, few of them, short pages
        _case("attention", "step_wide", dtype="fp16", heads=2, group=16, dim=256, page=16, batch=24, shortest=50, longest=6000),
        # drafted tokens being checked: several new tokens of each sequence
        _case("attention", "draft", batch=20, shortest=100, longest=6001, group=8, few=2, many=7, page=32),
        # whole prompts, packed, of different lengths
        _case("attention", "prompts", batch=4, shortest=300, longest=4096, few=0, many=0, lse=True),
        # one part of a long prompt behind those that the cache holds already
        _case("attention", "prompt_part", dtype="fp16", dim=64, shortest=32000, longest=32000, few=512, many=512),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(("write", "read", "attention", "attention", "attention"))
    kw = {"dtype": rng.choice(("bf16", "bf16", "fp16")), "dim": rng.choice((64, 128, 128, 256)), "page": rng.choice((16, 32, 64, 64, 80, 256)),
          "heads": rng.choice((1, 2, 3, 4, 8, 8)), "group": rng.choice((1, 2, 3, 4, 4, 5, 7, 8, 16)), "batch": log(1, 96)}
    wide = kw["heads"] * kw["dim"]
    if op != "attention":
        longest = max(1, min(log(1, 32768), int(2e7 / (wide * kw["batch"]))))
        all_new = op == "read" or rng.random() < 0.5
        return _case(op, shortest=log(1, longest), longest=longest, few=0 if all_new else 1, many=0 if all_new else rng.choice((1, 1, 5, 300)), **kw)
    kind = rng.choice(("step", "step", "draft", "prompt"))
    longest = max(1, min(log(1, 131072 if kind == "step" else 32768), int(1.3e8 / (wide * kw["batch"]))))
    few, many = {"step": (1, 1), "draft": (1, rng.randint(2, 24)), "prompt": (0, 0) if rng.random() < 0.6 else (1, log(25, 512))}[kind]
    rows = longest if many == 0 else many
    # the plain form's scores: batch * heads * group * rows * longest
    most = 4.0e10 / (kw["heads"] * kw["group"] * kw["dim"])
    while kw["batch"] * min(rows, longest) * longest > most:
        if kw["batch"] > 1:
            kw["batch"] = (kw["batch"] + 1) // 2
        else:
            longest = max(1, longest * 2 // 3)
        rows = longest if many == 0 else many
    return _case(op, shortest=log(1, longest), longest=longest, few=few, many=many, lse=rng.random() < 0.3, **kw)


def _lengths(case):
    """Tokens of each sequence, and how many of them are new: the same for every seed."""
    rng = random.Random(repr([(k, case[k]) for k in sorted(case) if k != "name"]))
    lo, hi = math.log(case["shortest"]), math.log(case["longest"])
    lens = [case["longest"]] + [int(round(math.exp(rng.uniform(lo, hi)))) for _ in range(case["batch"] - 1)]
    news = [n if case["many"] == 0 else min(n, rng.randint(case["few"], case["many"])) for n in lens]
    return lens, news


def _plan(case, g):
    """lens, pages and starts as a serving program has them: pages in any order, some of them used by no sequence."""
    lens, news = _lengths(case)
    page, device = case["page"], "cuda"
    width = -(-max(lens) // page)
    count = case["batch"] * width + 3
    pages = torch.randperm(count, generator=g, device=device)[:case["batch"] * width].view(case["batch"], width).to(torch.int32)
    starts = torch.tensor([0] + news, device=device).cumsum(0).to(torch.int32)
    return {"lens": torch.tensor(lens, dtype=torch.int32, device=device), "pages": pages, "starts": starts, "count": count, "rows": sum(news),
            "most": max(news), "longest": max(lens)}


def _places(s, steps, device):
    """For rows i < steps of every sequence, counted from its first new token: row number, position, and whether there is one."""
    new = (s["starts"][1:] - s["starts"][:-1]).long()
    i = torch.arange(steps, device=device)
    at = s["starts"][:-1].long()[:, None] + i
    position = (s["lens"].long() - new)[:, None] + i
    return at, position, i < new[:, None]


# The order of a granule's words: 8 codes a word, code e in bits 4 * (e // 2) + 16 * (e % 2).  Slabs of up to 128 channels.
# Keys: [slab][token][word % 4][word // 4]; values: [slab][token // 2][word % 8][token % 2][word // 8]; scales of keys
# [token][group], of values [slab][token // 2][group % 2][group // 2][token % 2].
def _to_words(codes):
    """[..., channels] to [..., channels / 8] 32-bit words."""
    at = torch.tensor([4 * (e // 2) + 16 * (e % 2) for e in range(8)], device=codes.device)
    w = ((codes.long().unflatten(-1, (-1, 8)) & 15) << at).sum(-1)
    return (w - ((w >> 31) << 32)).to(torch.int32)


def _from_words(words):
    at = torch.tensor([4 * (e // 2) + 16 * (e % 2) for e in range(8)], device=words.device, dtype=torch.int32)
    n = words.unsqueeze(-1) >> at & 15
    return (n - 16 * (n > 7)).flatten(-2)


def _quantize(x):
    """Codes and scales of [..., channels] fp32."""
    x = x.unflatten(-1, (-1, 32))
    top = x.abs().amax(-1)
    bits = (top / torch.full_like(top, 7.0)).view(torch.int32)   # by a number it would be a product with its reciprocal, and ties would be lost
    scale = (bits + 0x7ffff + (bits >> 20 & 1) & ~0xfffff).view(torch.float32)   # to four significant bits, ties to even
    scale = torch.where(top < 2.0 ** -100, 0.0, scale)
    codes = torch.where(scale[..., None] > 0, torch.round(x / torch.where(scale > 0, scale, 1.0)[..., None]), 0.0)
    return codes.flatten(-2).to(torch.int32), scale.to(torch.bfloat16)


def _granules(k, v):
    """Granules [..., 18 * dim] of keys and values [..., 16, dim], fp32."""
    dim = k.shape[-1]
    slabs = max(1, dim // 128)
    kc, ks = _quantize(k)
    vc, vs = _quantize(v)
    kw = _to_words(kc).unflatten(-1, (slabs, -1, 4)).movedim(-3, -4).transpose(-1, -2)            # slab, token, word % 4, word // 4
    vw = _to_words(vc).unflatten(-1, (slabs, -1, 8)).unflatten(-4, (8, 2))                        # pair, parity, slab, word // 8, word % 8
    vw = vw.movedim((-3, -5, -1, -4, -2), (-5, -4, -3, -2, -1))
    vs = vs.unflatten(-1, (slabs, -1, 2)).unflatten(-4, (8, 2))                                   # pair, parity, slab, group // 2, group % 2
    vs = vs.movedim((-3, -5, -1, -2, -4), (-5, -4, -3, -2, -1))
    lead = k.shape[:-2]
    parts = [p.contiguous().reshape(*lead, -1).view(torch.uint8) for p in (kw, vw, ks, vs)]
    return torch.cat(parts, -1)


def _values(granules):
    """Keys and values [..., 16, dim], fp32, of granules [..., 18 * dim]."""
    dim = granules.shape[-1] // 18
    slabs, part = max(1, dim // 128), min(dim, 128)
    lead = granules.shape[:-1]
    kw, vw, ks, vs = (granules[..., a * dim:b * dim] for a, b in ((0, 8), (8, 16), (16, 17), (17, 18)))
    kw = kw.contiguous().view(torch.int32).reshape(*lead, slabs, 16, 4, part // 32).transpose(-1, -2).movedim(-4, -3).reshape(*lead, 16, dim // 8)
    vw = vw.contiguous().view(torch.int32).reshape(*lead, slabs, 8, 8, 2, part // 64)
    vw = vw.movedim((-4, -2, -5, -1, -3), (-5, -4, -3, -2, -1)).reshape(*lead, 16, dim // 8)
    ks = ks.contiguous().view(torch.bfloat16).reshape(*lead, 16, dim // 32).float()
    vs = vs.contiguous().view(torch.bfloat16).reshape(*lead, slabs, 8, 2, part // 64, 2)
    vs = vs.movedim((-4, -1, -5, -2, -3), (-5, -4, -3, -2, -1)).reshape(*lead, 16, dim // 32).float()
    return (_from_words(kw).float().unflatten(-1, (-1, 32)) * ks[..., None]).flatten(-2), (_from_words(vw).float().unflatten(-1, (-1, 32)) * vs[..., None]).flatten(-2)


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _keys(g, *shape):
    """Keys have a few channels that are larger than the others, in every token; tokens differ in size."""
    k = _normal(g, *shape) * torch.exp(0.2 * _normal(g, shape[0], shape[1], 1))
    return k * (1.0 + 3.0 * (torch.rand(shape[1:], generator=g, device="cuda") < 0.03))


def _packed(g, case, rows):
    """Queries, keys and values as slices of one projection's output."""
    heads, group, dim = case["heads"], case["group"], case["dim"]
    qkv = torch.empty((rows, heads * (group + 2), dim), dtype=_TYPES[case["dtype"]], device="cuda")
    q, k, v = qkv.split([heads * group, heads, heads], 1)
    q.copy_(_normal(g, *q.shape))
    k.copy_(_keys(g, *k.shape))
    v.copy_(_normal(g, *v.shape))
    return q, k, v


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    state = dict(case, **_plan(case, g))
    state["q"], state["k"], state["v"] = _packed(g, case, state["rows"])
    shape = (state["count"], case["heads"], case["page"] // 16, 18 * case["dim"])
    state["cache"] = torch.zeros(shape, dtype=torch.uint8, device="cuda")
    if case["op"] != "write":   # what the cache holds, page by page, so that the values in fp32 need little memory
        for part in state["cache"].split(max(1, (1 << 26) // (case["heads"] * case["page"] * case["dim"]))):
            full = (part.shape[0], case["heads"], case["page"] // 16, 16, case["dim"])
            k = _keys(g, part.shape[0] * case["page"], case["heads"], case["dim"])
            k = k.view(part.shape[0], case["page"] // 16, 16, case["heads"], case["dim"]).movedim(3, 1)
            part.copy_(_granules(k, _normal(g, *full)))
    return state


def _run_own(s):
    import paper_2202_07471_b200 as sq

    if s["op"] == "attention":
        out = sq.squant_cache_attention(s["q"], s["cache"], s["lens"], s["pages"], s["starts"], most=s["most"], lse=s["lse"])
        return {"out": out[0], "lse": out[1]} if s["lse"] else {"out": out}
    if s["op"] == "write":
        sq.squant_cache_write(s["cache"], s["k"], s["v"], s["lens"], s["pages"], s["starts"])
    k, v = sq.squant_cache_read(s["cache"], s["lens"], s["pages"], s["starts"], s["rows"], dtype=_TYPES[s["dtype"]])
    return {"k": k, "v": v}


def _padded(s, steps):
    """Keys and values [batch, heads, steps, dim] of every sequence's first positions, fp32; behind its end, what the pages hold."""
    k, v = _values(s["cache"][s["pages"][:, :-(-steps // s["page"])].long()])   # batch, page, head, granule, token, dim
    return (x.movedim(2, 1).flatten(2, 4)[:, :, :steps] for x in (k, v))


def run(s):
    if own:
        return _run_own(s)
    dtype = _TYPES[s["dtype"]]
    at, position, there = _places(s, s["most"], s["lens"].device)
    if s["op"] == "write":
        # the granules that new tokens fall in, as they are, with the new tokens in their places
        page, place = torch.gather(s["pages"].long(), 1, (position.clamp(min=0) // s["page"]).clamp(max=s["pages"].shape[1] - 1))[there], position[there] % s["page"]
        granule = page * (s["page"] // 16) + place // 16
        which, back = torch.unique(granule, return_inverse=True)
        where = which // (s["page"] // 16), which % (s["page"] // 16)
        k, v = _values(s["cache"][where[0], :, where[1]])
        k[back, :, place % 16], v[back, :, place % 16] = s["k"][at[there]].float(), s["v"][at[there]].float()
        s["cache"][where[0], :, where[1]] = _granules(k, v)
    if s["op"] != "attention":
        page, place = torch.gather(s["pages"].long(), 1, (position.clamp(min=0) // s["page"]).clamp(max=s["pages"].shape[1] - 1))[there], position[there] % s["page"]
        k, v = _values(s["cache"][page, :, place // 16])
        pick = torch.arange(page.numel(), device=page.device)
        return {"k": k[pick, :, place % 16].to(dtype), "v": v[pick, :, place % 16].to(dtype)}
    k, v = _padded(s, s["longest"])
    heads, group = s["heads"], s["group"]
    q = s["q"][at.clamp(max=s["rows"] - 1)].float().unflatten(2, (heads, group)).movedim(1, 3)           # batch, head, group, row, dim
    scores = torch.matmul(q.flatten(2, 3), k.transpose(-1, -2)).unflatten(2, (group, -1))
    seen = torch.arange(s["longest"], device=k.device) <= position[:, None, None, :, None]
    scores = torch.where(seen, scores * (1.0 / math.sqrt(s["dim"])), -math.inf)
    top = scores.amax(-1, keepdim=True).clamp(min=-3e38)
    p = torch.exp(scores - top)
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p.flatten(2, 3), v).unflatten(2, (group, -1)) / torch.where(total > 0, total, 1.0)
    out = out.movedim(3, 1).flatten(2, 3)[there].to(dtype)
    if not s["lse"]:
        return {"out": out}
    return {"out": out, "lse": (top + torch.log(total)).squeeze(-1).movedim(3, 1).flatten(2, 3)[there]}


def exact(case, seed):
    """The operators' definition in 64 bits, sequence by sequence, written apart from the forms above."""
    lens, news = _lengths(case)
    heads, group, dim, page = case["heads"], case["group"], case["dim"], case["page"]
    pairs = sum(m * (2 * n - m + 1) / 2 for n, m in zip(lens, news))
    if case["op"] == "attention" and pairs * heads * group * dim > 4e12:
        return None
    s = prepare(case, seed)
    f64 = torch.float64

    def stood_for(x):   # what 32 channels' codes and scale stand for
        x = x.to(f64).reshape(*x.shape[:-1], -1, 32)
        step = x.abs().amax(-1, keepdim=True)
        step = step / torch.full_like(step, 7.0)
        unit = torch.ldexp(torch.ones_like(step), torch.frexp(step).exponent - 4)
        step = torch.round(step / unit) * unit
        return (torch.round(x / torch.where(step > 0, step, torch.ones_like(step))) * step).flatten(-2)

    if case["op"] == "write":
        return {"k": stood_for(s["k"]), "v": stood_for(s["v"])}

    def word_values(raw, scales, words, groups):
        """raw [..., words of 4 bytes] in the granule's order; words, groups: its place for each token's word and group, [16, n]."""
        b = raw.to(torch.int64).reshape(*raw.shape[:-1], -1, 4)[..., words.flatten(), :]
        b = torch.stack([b[..., 2 * (e % 2) + e // 4] >> 4 * (e // 2 % 2) & 15 for e in range(8)], -1)   # code e of a word
        code = ((b + 8) % 16 - 8).to(f64).reshape(*raw.shape[:-1], 16, dim)
        s16 = scales.contiguous().view(torch.bfloat16).to(f64)[..., groups.flatten()].reshape(*raw.shape[:-1], 16, dim // 32)
        return code * s16.repeat_interleave(32, -1)

    slab = min(dim, 128)
    per_word, per_group = slab // 8, slab // 32
    places = [torch.zeros((16, dim // n), dtype=torch.int64, device="cuda") for n in (8, 8, 32, 32)]
    for t in range(16):
        for w in range(dim // 8):
            a, r = divmod(w, per_word)
            places[0][t, w] = a * 16 * per_word + t * per_word + r % 4 * (per_word // 4) + r // 4
            places[1][t, w] = a * 16 * per_word + t // 2 * 2 * per_word + r % 8 * 2 * (per_word // 8) + t % 2 * (per_word // 8) + r // 8
        for n in range(dim // 32):
            a, r = divmod(n, per_group)
            places[2][t, n] = t * (dim // 32) + n
            places[3][t, n] = a * 16 * per_group + t // 2 * 2 * per_group + r % 2 * per_group + r // 2 * 2 + t % 2

    def sequence(b, first, last):
        """Keys and values [tokens, heads, dim] of positions first .. last."""
        g = s["cache"][s["pages"][b, first // page:-(-last // page)].long()].movedim(1, 2).reshape(-1, heads, 18 * dim)
        k = word_values(g[..., :8 * dim], g[..., 16 * dim:17 * dim], places[0], places[2])
        v = word_values(g[..., 8 * dim:16 * dim], g[..., 17 * dim:], places[1], places[3])
        skip = first - first // page * page
        return (x.transpose(1, 2).reshape(-1, heads, dim)[skip:skip + last - first] for x in (k, v))

    if case["op"] == "read":
        parts = [tuple(sequence(b, n - m, n)) for b, (n, m) in enumerate(zip(lens, news))]
        return {"k": torch.cat([p[0] for p in parts]), "v": torch.cat([p[1] for p in parts])}
    out = torch.empty((sum(news), heads * group, dim), dtype=f64, device="cuda")
    lse = torch.empty((sum(news), heads * group), dtype=f64, device="cuda")
    row = 0
    for b, (n, m) in enumerate(zip(lens, news)):
        k, v = sequence(b, 0, n)
        hidden = torch.arange(n, device="cuda")[None, :] > torch.arange(n - m, n, device="cuda")[:, None]
        for h in range(heads * group):
            z = (s["q"][row:row + m, h].to(f64) @ k[:, h // group].T / math.sqrt(dim)).masked_fill_(hidden, -math.inf)
            lse[row:row + m, h] = torch.logsumexp(z, -1)
            out[row:row + m, h] = torch.softmax(z, -1) @ v[:, h // group]
        row += m
    return {"out": out, "lse": lse} if case["lse"] else {"out": out}


def work(case):
    lens, news = _lengths(case)
    heads, group, dim = case["heads"], case["group"], case["dim"]
    stored = heads * 18 * dim / 16   # bytes of a token
    if case["op"] == "write":        # read, stored, read back and returned
        return {"bytes": sum(news) * 2 * (4 * heads * dim + stored), "flops": 0}
    if case["op"] == "read":
        return {"bytes": sum(news) * (4 * heads * dim + stored), "flops": 0}
    pairs = sum(m * (2 * n - m + 1) / 2 for n, m in zip(lens, news))   # of a row and a token that it sees
    return {"bytes": sum(lens) * stored + sum(news) * heads * group * (4 * dim + 4 * case["lse"]), "flops": 4.0 * pairs * heads * group * dim}
