"""The key/value cache on the GPU: writing, reading, attention, against plain 64-bit forms."""
import math

import pytest
import torch

import paper_2202_07471_b200 as sq
from cache_cases import Batch, attention, filled, gen, parts, scale_of, stored, values

pytestmark = pytest.mark.gpu
BF16, FP16 = torch.bfloat16, torch.float16


def inputs(rows, heads, dim, dtype, seed, pad=0, head_pad=0):
    """Keys or values [rows, heads, dim], slices of a wider buffer where there is a pad."""
    wide = torch.randn((rows, heads, dim + head_pad), generator=gen(seed), device="cuda").to(dtype)
    if pad:
        wide = torch.cat((wide, torch.full((rows, pad, dim + head_pad), 7.0, dtype=dtype, device="cuda")), 1)
    return wide[:, :heads, :dim]


def same(a, b):
    """Equal values, NaN in the same places."""
    a, b = a.double(), b.double()
    return a.shape == b.shape and bool(((a == b) | (a.isnan() & b.isnan())).all())


# ---- write and read

@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("heads,page,pad,head_pad", [(1, 16, 0, 0), (3, 48, 2, 0), (8, 64, 0, 0), (5, 128, 1, 3), (2, 32, 0, 8)])
def test_written_values_are_the_formula_s(dim, dtype, heads, page, pad, head_pad):
    batch = Batch([40, 1, 0, 17, 130], [40, 1, 0, 5, 33], page, seed=3)
    cache = sq.alloc_cache(batch.page_count, heads, dim, page_size=page)
    k, v = inputs(batch.rows, heads, dim, dtype, 1, pad, head_pad), inputs(batch.rows, heads, dim, dtype, 2, pad, head_pad)
    version = cache._version
    assert sq.squant_cache_write(cache, k, v, *batch.args) is None and cache._version > version
    kc, ks, vc, vs = parts(cache)
    kf, vf = values(cache)
    touched = torch.zeros(cache.shape[0], page, dtype=torch.bool)
    for b, n in enumerate(batch.lens_list):
        span = batch.rows_of(b)
        for full, x, scales in ((kf, k, ks), (vf, v, vs)):
            got = batch.sequence(full, b)[n - len(span):]
            want = x[span.start:span.stop]
            assert same(got, stored(want))
            assert same(batch.sequence(scales, b)[n - len(span):], scale_of(want))
        for p in range(n - len(span), n):
            touched[batch.pages_list[b, p // page], p % page] = True
    untouched = ~touched.cuda()[:, None, :, None]
    assert not (kc * untouched).any() and not (vc * untouched).any() and not (ks * untouched).any() and not (vs * untouched).any()
    # and back, in both types: exact in bf16, rounded once in fp16
    for out in (BF16, FP16):
        rk, rv = sq.squant_cache_read(cache, *batch.args, batch.rows, dtype=out)
        assert rk.dtype == out and same(rk, stored(k).to(out)) and same(rv, stored(v).to(out))
    buf = inputs(batch.rows, heads, dim, FP16, 9, pad + 1, head_pad), inputs(batch.rows, heads, dim, FP16, 9, pad + 1, head_pad)
    got = sq.squant_cache_read(cache, *batch.args, batch.rows, k=buf[0], v=buf[1])
    assert got[0] is buf[0] and same(buf[0], stored(k).to(FP16)) and same(buf[1], stored(v).to(FP16))


def test_every_tie_and_magnitude():
    """All ratios of two bfloat16 numbers' mantissas near a tie of scale or code: largest values of every mantissa, values on and next to halves of a step."""
    rows = []
    for m in range(128):
        for exponent in (-90, -20, 0, 9, 100):
            top = (1 + m / 128) * 2.0 ** exponent
            s = float(scale_of(torch.full((32,), top, dtype=torch.float64))[0])
            x = torch.empty(32, dtype=torch.float64)
            x[0] = top if m % 2 else -top
            x[1:15] = torch.arange(-7, 7, dtype=torch.float64).add(0.5) * s
            x[15:31] = torch.arange(-8, 8, dtype=torch.float64).mul(s) * (1 + 2.0 ** -8)
            x[31] = 0.0
            rows.append(x.clamp(-abs(top), abs(top)))
    x = torch.stack(rows).view(-1, 2, 32).flatten(1).to(BF16).cuda()[:, None, :]
    n = x.shape[0]
    batch = Batch([n], [n], 64)
    cache = sq.alloc_cache(batch.page_count, 1, 64)
    sq.squant_cache_write(cache, x, -x, *batch.args)
    k, v = sq.squant_cache_read(cache, *batch.args, n)
    assert same(k, stored(x)) and same(v, stored(-x))
    kc, _, vc, _ = parts(cache)
    assert kc.abs().max() == 7 and vc.abs().max() == 7


def test_values_without_a_number_small_and_large_ones():
    x = torch.randn((6, 1, 128), generator=gen(1), device="cuda").to(BF16)
    x[0, 0, 3], x[1, 0, 40], x[2, 0, 127] = math.inf, -math.inf, math.nan
    x[3] = 0
    x[4, 0, :32], x[4, 0, 32:64], x[4, 0, 64:96] = 2.0 ** -101, 2.0 ** -100, 2.0 ** 120
    x[5, 0, :32] = 1.3e36
    batch = Batch([6], [6], 16)
    cache = sq.alloc_cache(batch.page_count, 1, 128, page_size=16)
    sq.squant_cache_write(cache, x, x.flip(0), *batch.args)
    k, v = sq.squant_cache_read(cache, *batch.args, 6)
    want = stored(x)
    assert same(k, want) and same(v, want.flip(0))
    assert k[0, 0, :32].isnan().all() and not k[0, 0, 32:].isnan().any() and k[4, 0, 64:96].isnan().all() and (k[4, 0, :32] == 0).all() and not (k[4, 0, 32:64] == 0).any()


def test_rows_without_a_place():
    """Rows behind the last sequence, before a sequence's first position, in pages that are not there; starts, lengths that lead nowhere."""
    heads, dim, page = 2, 64, 16
    batch = Batch([20, 3, 40], [4, 5, 40], page, extra_rows=6)
    batch.pages[2, 1] = batch.page_count          # not there
    batch.pages[0, 0] = -1                        # not read: position 16 to 19
    cache = sq.alloc_cache(batch.page_count, heads, dim, page_size=page)
    x = inputs(batch.rows, heads, dim, BF16, 1)
    sq.squant_cache_write(cache, x, x, *batch.args)
    k = torch.full((batch.rows, heads, dim), 5.0, dtype=BF16, device="cuda")
    v = k.clone()
    sq.squant_cache_read(cache, *batch.args, batch.rows, k=k, v=v)
    want = stored(x)
    want[4:6] = 0                # sequence 1 has five rows and three positions
    want[9 + 16:9 + 32] = 0
    want[49:] = 5
    assert same(k, want) and same(v, want)
    # what the arrays hold may be anything
    before = cache.clone()
    for lens, starts in (([-5, -1, -2 ** 31], [0, 4, 9, 49]), ([20, 3, 40], [-7, -3, -2, -1]), ([20, 3, 40], [100, 200, 300, 2 ** 31 - 1]), ([20, 3, 40], [60, 40, 20, 0])):
        sq.squant_cache_write(cache, x, x, torch.tensor(lens, dtype=torch.int32, device="cuda"), batch.pages, torch.tensor(starts, dtype=torch.int32, device="cuda"))
    assert torch.equal(cache, before)
    lens = torch.full((3,), 2 ** 31 - 1, dtype=torch.int32, device="cuda")   # cut to what pages covers: 48 positions
    rk, _ = sq.squant_cache_read(cache, lens, batch.pages, batch.starts, batch.rows)
    assert same(rk[:4], values(cache)[0][batch.pages_list[0, 2]].transpose(0, 1)[12:16])
    assert sq.squant_device_status() is None


def test_many_sequences_find_their_rows():
    """More sequences than one round of the search takes, many of them without rows."""
    g = torch.Generator().manual_seed(5)
    lens = torch.randint(0, 40, (3000,), generator=g).tolist()
    news = [min(n, int(torch.randint(0, 4, (1,), generator=g))) for n in lens]
    batch = Batch(lens, news, 16)
    cache = sq.alloc_cache(batch.page_count, 1, 64, page_size=16)
    x = inputs(batch.rows, 1, 64, BF16, 1)
    sq.squant_cache_write(cache, x, -x, *batch.args)
    k, v = sq.squant_cache_read(cache, *batch.args, batch.rows)
    assert same(k, stored(x)) and same(v, -stored(x))
    kf, _ = values(cache)
    for b in (0, 1, 31, 32, 33, 1023, 1024, 2999):
        n = lens[b]
        assert same(batch.sequence(kf, b)[n - news[b]:], stored(x[batch.rows_of(b).start:batch.rows_of(b).stop]))


# ---- attention

# What the kernels round:
#   the output, by half a step of its type: 2^-8 (2^-11) of |out|, in fp16 at least 2^-25, half its smallest number
#   with more than eight rows the weights of the product with the values, by half a step: the output, an average of the values, moves by at most 2^-8 (2^-11) of sum p |v|.  In
#   fp16 a weight (the largest is at least 1) is off by at least 2^-25 too, also where what is left over goes through a second product: 2^-25 sum |v| in all
#   scores: their exponents s log2(e) - m in fp32, and the sums of products, of which the tensor cores cut off 2^-23 of the largest at most 16 + 3 times: 2^-18 |s| of each
#   weight, with |lse| for the largest |s|.  All other fp32 operations: 2^-16 of sum p |v|
#   weights that are lost: exponentials below 2^-126 are 0, and a row's maximum so far, against which a part of it was summed, may lie 2^64 below its weights (2^14 in fp16) before it
#   is replaced: weights below 2^(64 - 126) of the row's largest, which is at least 1: 2^-62 max |v| for each position
# fp16 values are those that squant_cache_read returns in fp16: exact for the sizes here.
def check_attention(out, lse, q, batch, cache, scale=None, rounded_p=True):
    want, want_lse = attention(q, batch, cache, scale)
    size = attention_sizes(q, batch, cache, scale)
    step = torch.finfo(out.dtype).eps / 2
    inside = torch.zeros(q.shape[0], dtype=torch.bool, device="cuda")
    inside[:sum(batch.news)] = True
    slack = step * want.abs() + (step * rounded_p + 2.0 ** -16 + 2.0 ** -18 * want_lse.abs().clamp(max=1e6)[..., None]) * size + 2.0 ** -62 * max(batch.lens_list) * float(values(cache)[1].nan_to_num(0).abs().max())
    if out.dtype == FP16:
        slack = slack + 2.0 ** -25 * (1 + max(batch.lens_list) * float(values(cache)[1].nan_to_num(0).abs().max()))
    off = (out.double() - want).abs()
    bad = (off > slack) & inside[:, None, None]
    assert not bad.any(), (int(bad.sum()), float((off / slack)[inside].max()))
    if lse is not None:
        none = want_lse == -math.inf
        assert torch.equal((lse == -math.inf) & inside[:, None], none & inside[:, None])
        ok = inside[:, None] & ~none
        assert ((lse.double() - want_lse).abs()[ok] <= 2.0 ** -17 * (1 + want_lse.abs()[ok])).all()


def attention_sizes(q, batch, cache, scale=None):
    """sum p |v| of every output."""
    flipped = _with_sizes(cache)
    return attention(q, batch, flipped, scale)[0]


def _with_sizes(cache):
    """The same keys, the values' magnitudes (codes made positive)."""
    from cache_cases import places
    dim = cache.shape[3] // 18
    out = cache.clone()
    part = out[..., 8 * dim:16 * dim].to(torch.int32)
    low, high = part & 15, part >> 4
    low, high = torch.where(low > 7, 16 - low, low), torch.where(high > 7, 16 - high, high)
    out[..., 8 * dim:16 * dim] = (low | high << 4).to(torch.uint8)
    assert places(dim)["v"].min() == 8 * dim
    return out


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("heads,group,page,lens", [(1, 1, 16, [1]), (2, 8, 64, [5, 0, 33, 64]), (3, 5, 48, [1000, 17, 16, 31, 32]), (8, 4, 64, [700]), (1, 16, 32, [260, 1]),
                                                  (2, 7, 16, [4099, 1, 513]), (4, 3, 128, [257, 255, 256, 0])])
def test_single_tokens(dim, dtype, heads, group, page, lens):
    batch = Batch(lens, [1] * len(lens), page, seed=1)
    cache = filled(batch, heads, dim, 5)
    q = inputs(batch.rows, heads * group, dim, dtype, 3)
    for starts in (None, batch.starts):
        out, lse = sq.squant_cache_attention(q, cache, batch.lens, batch.pages, starts, most=1, lse=True)
        check_attention(out, lse, q, batch, cache, rounded_p=group > 8)
    assert sq.squant_device_status() is None


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("heads,group,page,lens,news", [
    (2, 1, 16, [9, 40, 0, 7], [9, 5, 0, 7]), (1, 4, 64, [70, 33, 2], [2, 2, 2]), (2, 3, 32, [100, 3, 65], [20, 5, 1]), (1, 8, 48, [300, 290], [16, 17]),
    (3, 2, 16, [64, 65, 1], [64, 65, 1]), (1, 5, 128, [500], [131])])
@pytest.mark.parametrize("hint", [False, True])
def test_several_tokens(dim, dtype, heads, group, page, lens, news, hint):
    """Causal masks inside units, rows before the first position, padded rows, rows of several tiles."""
    batch = Batch(lens, news, page, seed=2, extra_rows=3)
    cache = filled(batch, heads, dim, 15)
    q = inputs(batch.rows, heads * group, dim, dtype, 4, pad=1)
    out = torch.full((batch.rows, heads * group, dim), 3.0, dtype=dtype, device="cuda")
    got, lse = sq.squant_cache_attention(q, cache, *batch.args, most=max(news) if hint else 0, lse=True, out=out, scale=0.11)
    assert got is out and (out[sum(news):] == 3).all()
    check_attention(out, lse, q, batch, cache, 0.11)
    assert sq.squant_device_status() is None


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("news,most", [(1, 1), (2, 2), (40, 0)])
@pytest.mark.parametrize("rise", [5.0, 30.0, 200.0])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_scores_that_grow(dtype, dim, news, most, rise, sign):
    """Scores reach far beyond all before, several times, in the middle of what is taken at once; with a negative scale too."""
    heads, group, page, n = 2, 4, 32, 700
    batch = Batch([n, 300], [news, news], page, seed=4)
    shape = (batch.page_count, heads, page // 16, 16, dim)
    k = torch.randn(shape, generator=gen(1), device="cuda") * 0.3
    v = torch.randn(shape, generator=gen(2), device="cuda")
    direction = torch.randn(dim, generator=gen(3), device="cuda").sign()
    for b in range(2):
        for step, p in enumerate((3, 70, 130, 165, 217, 290, 450, 455, 640)):
            if p < batch.lens_list[b]:
                k[batch.pages_list[b, p // page], :, p % page // 16, p % 16] += direction * (step + 1) * rise / 9 / dim ** 0.5
    from cache_cases import pack
    cache = pack(k.to(dtype), v.to(dtype))
    q = (inputs(batch.rows, heads * group, dim, dtype, 7).float() * 0.3 + direction).to(dtype)
    out, lse = sq.squant_cache_attention(q, cache, *batch.args, most=most, lse=True, scale=sign * 1.0)
    check_attention(out, lse, q, batch, cache, sign * 1.0)
