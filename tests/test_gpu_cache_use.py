"""The key/value cache as a program uses it: with the linear layers, on streams, in graphs, with bad pages, in its checked build."""
import math

import pytest
import torch

import paper_2202_07471_b200 as sq
from cache_cases import Batch, attention, filled, gen, pack, stored, values
from paper_2202_07471_b200 import binding, build as lib_build, cache as cache_module
from test_gpu_cache import BF16, FP16, check_attention, inputs, same

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_a_layer_s_prompt_and_steps(dtype):
    """A layer on quantized weights: projection, keys and values into the cache, attention, projection back - a prompt, then token by token; the rows are those of one
    pass over all tokens at once."""
    heads, group, dim, page, features = 2, 4, 64, 16, 512
    w1 = torch.randn((heads * (group + 2) * dim, features), generator=gen(1), device="cuda") / features ** 0.5
    w2 = torch.randn((features, heads * group * dim), generator=gen(2), device="cuda") / (heads * group * dim) ** 0.5
    q1, q2 = sq.alloc_outputs(w1, pack_int4=True), sq.alloc_outputs(w2, pack_int4=True)
    sq.squant_quantize_model([q1, q2], bits=4, flags=sq.FLAG_NARROW_RANGE | sq.FLAG_PACK_INT4)
    x = torch.randn((90, features), generator=gen(3), device="cuda").to(dtype)

    def layer(rows, cache, lens, pages, starts, most):
        qkv = sq.squant_linear(rows, q1.codes, q1.scales, pack_int4=True).view(-1, heads * (group + 2), dim)
        q, k, v = qkv.split([heads * group, heads, heads], 1)
        sq.squant_cache_write(cache, k, v, lens, pages, starts)
        out = sq.squant_cache_attention(q, cache, lens, pages, starts, most=most)
        return sq.squant_linear(out.flatten(1), q2.codes, q2.scales, residual=rows, pack_int4=True)

    whole = Batch([50, 40], [50, 40], page)
    cache = sq.alloc_cache(whole.page_count, heads, dim, page_size=page)
    want = layer(x, cache, *whole.args, 50)
    again = sq.alloc_cache(whole.page_count, heads, dim, page_size=page)
    prompt = Batch([44, 30], [44, 30], page)
    first = layer(torch.cat((x[:44], x[50:80])), again, prompt.lens, whole.pages, prompt.starts, 44)
    got = torch.empty_like(want)
    got[:44], got[50:80] = first[:44], first[44:]
    for i in range(6):
        lens = torch.tensor([45 + i, 31 + i], dtype=torch.int32, device="cuda")
        got[[44 + i, 80 + i]] = layer(x[[44 + i, 80 + i]], again, lens, whole.pages, None, 1)
    got[86:] = layer(x[86:], again, torch.tensor([50, 40], dtype=torch.int32, device="cuda"), whole.pages, torch.tensor([0, 0, 4], dtype=torch.int32, device="cuda"), 4)
    # projections and attention round in other places than the whole pass does: a few steps of the type, of values near 1
    assert (got.double() - want.double()).abs().max() <= 16 * torch.finfo(dtype).eps * want.abs().max()
    assert sq.squant_device_status() is None


def test_native_calls_are_the_binding_s(monkeypatch):
    batch = Batch([70, 5, 33], [7, 1, 3], 16)
    for dtype in (BF16, FP16):
        k, v, q = (inputs(batch.rows, h, 128, dtype, 3 + h, pad=1) for h in (2, 2, 6))
        got = []
        for native in (True, False):
            if not native:
                monkeypatch.setattr(cache_module, "_native", lambda: None)
            cache = filled(batch, 2, 128, 4)
            version = cache._version
            assert sq.squant_cache_write(cache, k, v, *batch.args) is None and cache._version == version + 1
            out = torch.zeros_like(q.contiguous())
            res = sq.squant_cache_attention(q, cache, *batch.args, lse=True, out=out, most=7)
            assert res[0] is out and out._version == 1
            got.append((cache, out, res[1], *sq.squant_cache_read(cache, *batch.args, batch.rows, dtype=dtype), sq.squant_cache_attention(q, cache, *batch.args, scale=-0.3)))
        monkeypatch.undo()
        assert binding._marshal is None or cache_module._native() is not None
        assert all(torch.equal(a, b) for a, b in zip(*got))
    # what the native calls leave to the binding has its errors
    for bad in (lambda: sq.squant_cache_write(cache, k, v[:-1], *batch.args), lambda: sq.squant_cache_attention(q[:, :5], cache, *batch.args),
                lambda: sq.squant_cache_attention(q.float(), cache, *batch.args), lambda: sq.squant_cache_read(cache, batch.lens.long(), batch.pages, batch.starts, 3),
                lambda: sq.squant_cache_attention(q, cache, *batch.args, most=-1), lambda: sq.squant_cache_attention(q, cache.cpu(), *batch.args)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(sq.SquantError):
        sq.squant_cache_attention(q, cache, *batch.args, scale=math.nan)


def test_streams_and_two_calls_at_once():
    batch = Batch([3000, 70, 900], [1, 1, 1], 64)
    cache = filled(batch, 4, 128, 7)
    q = inputs(3, 16, 128, BF16, 8)
    want = sq.squant_cache_attention(q, cache, *batch.args, most=1)
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    outs = []
    for _ in range(20):
        for s in streams:
            outs.append(sq.squant_cache_attention(q, cache, *batch.args, most=1, stream=s))
            with torch.cuda.stream(s):
                outs.append(sq.squant_cache_attention(q, cache, *batch.args, most=1))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)
    side = torch.cuda.Stream()
    k, v = sq.squant_cache_read(cache, *batch.args, 3, stream=side)
    side.synchronize()
    assert torch.equal(k, sq.squant_cache_read(cache, *batch.args, 3)[0])


@pytest.mark.parametrize("most", [1, 0])
def test_a_captured_step_is_replayed_with_other_lengths(most):
    heads, group, dim, page, batch = 2, 4 if most else 12, 128, 32, 5   # with 60 rows of a sequence possible, the kernel for prompts
    room = Batch([400] * batch, [1] * batch, page)
    cache = filled(room, heads, dim, 3)
    lens, q = torch.ones(batch, dtype=torch.int32, device="cuda"), inputs(batch, heads * group, dim, BF16, 4)
    k, v = inputs(batch, heads, dim, BF16, 5), inputs(batch, heads, dim, BF16, 6)

    def step():
        sq.squant_cache_write(cache, k, v, lens, room.pages)
        return sq.squant_cache_attention(q, cache, lens, room.pages, room.starts if most == 0 else None, most=most, lse=True)

    step()
    torch.cuda.synchronize()
    graph, second = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = step()
    with torch.cuda.graph(second, pool=graph.pool()):
        out2, _ = step()
    for i, values_ in enumerate(([1, 400, 33, 32, 31], [400, 399, 1, 2, 3], [64] * 5, [0, -3, 5, 1000, 7])):
        lens.copy_(torch.tensor(values_, dtype=torch.int32))
        k.copy_(inputs(batch, heads, dim, BF16, 50 + i))
        for g, o in ((graph, out), (second, out2), (graph, out)):
            g.replay()
            torch.cuda.synchronize()
            plain = Batch([max(0, min(x, 416)) for x in values_], [1] * batch, page)
            plain.pages_list = room.pages_list
            check_attention(o, lse if o is out else None, q, plain, cache)


def test_values_without_a_number_in_hidden_places():
    """A later token's infinities are not seen by the rows before it, and pages behind the end may hold anything."""
    heads, group, dim, page = 2, 2, 128, 16
    for news, most in ((4, 4), (40, 0), (40, 2), (200, 0)):
        batch = Batch([300, 210], [news, news], page, seed=2)
        cache = filled(batch, heads, dim, 9)
        q = inputs(batch.rows, heads * group, dim, BF16, 4)
        clean = sq.squant_cache_attention(q, cache, *batch.args, most=most).clone()
        for t in range(302, 304):   # behind the end, in the last page
            cache[batch.pages_list[0, t // page], :, t % page // 16] = cache[batch.pages_list[0, t // page], :, t % page // 16]
        last = batch.pages_list[0, 299 // page]
        k = torch.randn((heads, 1, 16, dim), device="cuda", generator=gen(5)).to(BF16)
        v = k.clone()
        kf, vf = (batch.sequence(x, 0, 304).to(BF16) for x in values(cache))
        kk, vv = kf[288:304].transpose(0, 1).clone(), vf[288:304].transpose(0, 1).clone()
        kk[:, 12:], vv[:, 12:] = math.nan, math.inf          # positions 300 to 303: behind the end
        vv[0, 11, 40] = math.inf                              # position 299, the last one: group 1 of head 0
        kk[1, 11, 3] = math.nan
        cache[last, :, 0] = pack(kk, vv)
        got = sq.squant_cache_attention(q, cache, *batch.args, most=most)
        row = news - 1
        assert torch.equal(got[:row], clean[:row]) and torch.equal(got[news:], clean[news:])
        assert got[row, :group, 32:64].isnan().all() and not got[row, :group, :32].isnan().any() and not got[row, :group, 64:].isnan().any() and got[row, group:].isnan().all()


@pytest.mark.parametrize("news,most", [(1, 1), (3, 3), (30, 0)])
def test_pages_that_are_not_there(news, most):
    """Their positions are not attended to; a sequence without any page that is there sees nothing."""
    heads, group, dim, page = 2, 4, 64, 32
    batch = Batch([200, 64, 97], [news, news, news], page, extra_rows=2)
    cache = filled(batch, heads, dim, 3)
    q = inputs(batch.rows, heads * group, dim, BF16, 4)
    pages = batch.pages.clone()
    pages[0, 2], pages[0, 3], pages[1, :] = -1, batch.page_count, 2 ** 31 - 1
    out = torch.full(q.shape, 9.0, dtype=BF16, device="cuda")
    got, lse = sq.squant_cache_attention(q, cache, batch.lens, pages, batch.starts, most=most, lse=True, out=out)
    k_full, v_full = values(cache)
    for b, gone in ((0, range(64, 128)), (1, range(0, 64)), (2, ())):
        k, v = batch.sequence(k_full, b), batch.sequence(v_full, b)
        for i, row in enumerate(batch.rows_of(b)):
            seen = [t for t in range(batch.lens_list[b] - news + i + 1) if t not in gone]
            if not seen:
                assert not got[row].any() and (lse[row] == -math.inf).all()
                continue
            s = torch.einsum("hd,jhd->hj", q[row].double(), k[seen].repeat_interleave(group, 1)) / dim ** 0.5
            want = torch.einsum("hj,jhd->hd", s.softmax(-1), v[seen].repeat_interleave(group, 1))
            size = torch.einsum("hj,jhd->hd", s.softmax(-1), v[seen].abs().repeat_interleave(group, 1))
            assert ((got[row].double() - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -8 + 2.0 ** -15) * size).all()
    assert (out[3 * news:] == 9).all() and sq.squant_device_status() is None


def test_a_cache_beyond_32_bits():
    heads, dim, page = 8, 128, 64
    pages = 80_000                                    # 5.9 GB
    cache = sq.alloc_cache(pages, heads, dim, page_size=page)
    batch = Batch([150, 70], [150, 70], page)
    batch.pages_list = torch.tensor([[79_999, 3, 60_000], [79_998, 70_001, 5]])
    batch.pages = batch.pages_list.to(torch.int32).cuda()
    k, v, q = (inputs(batch.rows, h, dim, BF16, h) for h in (heads, heads, 2 * heads))
    sq.squant_cache_write(cache, k, v, batch.lens, batch.pages, batch.starts)
    rk, rv = sq.squant_cache_read(cache, batch.lens, batch.pages, batch.starts, batch.rows)
    assert same(rk, stored(k)) and same(rv, stored(v))
    small = sq.alloc_cache(6, heads, dim, page_size=page)
    table = torch.arange(6, dtype=torch.int32, device="cuda").view(2, 3)
    sq.squant_cache_write(small, k, v, batch.lens, table, batch.starts)
    for most in (0, 2):
        a = sq.squant_cache_attention(q, cache, batch.lens, batch.pages, batch.starts, most=most)
        assert torch.equal(a, sq.squant_cache_attention(q, small, batch.lens, table, batch.starts, most=most))


def test_many_sequences_short_and_long():
    """More sequences than one round of the work's division takes, most of them short, one long; none at all."""
    g = torch.Generator().manual_seed(3)
    lens = torch.randint(1, 60, (300,), generator=g).tolist()
    lens[170] = 5000
    news = [min(n, int(torch.randint(0, 3, (1,), generator=g))) for n in lens]
    batch = Batch(lens, news, 16)
    cache = filled(batch, 2, 64, 3)
    q = inputs(batch.rows, 6, 64, BF16, 5)
    outs = [sq.squant_cache_attention(q, cache, *batch.args, most=most, lse=True) for most in (2, 4, 0)]
    for i, (out, lse) in enumerate(outs):
        check_attention(out, lse, q, batch, cache)
        again = sq.squant_cache_attention(q, cache, *batch.args, most=(2, 4, 0)[i], lse=True)
        assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
    none = torch.zeros(301, dtype=torch.int32, device="cuda")
    keep = torch.full(q.shape, 2.0, dtype=BF16, device="cuda")
    for most in (2, 0):
        sq.squant_cache_attention(q, cache, batch.lens, batch.pages, none, most=most, out=keep)
    assert (keep == 2).all()
    empty = sq.alloc_cache(0, 2, 64)
    table = torch.zeros((2, 0), dtype=torch.int32, device="cuda")
    lens2 = torch.tensor([4, 0], dtype=torch.int32, device="cuda")
    assert not sq.squant_cache_attention(q[:2], empty, lens2, table).any()
    sq.squant_cache_write(empty, q[:2, :2], q[:2, :2], lens2, table)
    assert not sq.squant_cache_read(empty, lens2, table, None, 2)[0].any()


# ---- checked build, failure path

@pytest.fixture
def checked_build():
    sq.use_library(lib_build.LIB_DEBUG)
    try:
        yield
    finally:
        sq.squant_debug_linear_wait_limit(-1)
        sq.use_library(None)


def _status():
    try:
        sq.squant_device_status()
        return 0
    except sq.SquantError as e:
        return e.code


SHAPES = [(64, 2, 4, 16, [5, 0, 33, 700], [3, 0, 33, 2]), (128, 3, 5, 48, [1000, 17, 16, 31], [1, 1, 1, 1]), (128, 2, 4, 64, [600, 300], [600, 9]), (256, 1, 7, 32, [333, 90], [100, 1]),
          (64, 8, 8, 128, [257, 255, 256], [17, 1, 40]), (256, 2, 16, 16, [50, 600], [1, 1])]


@pytest.mark.parametrize("dim,heads,group,page,lens,news", SHAPES)
def test_indices_stay_in_bounds(dim, heads, group, page, lens, news):
    batch = Batch(lens, news, page, extra_rows=1)
    k, v, q = (inputs(batch.rows, h, dim, BF16, h + 1, pad=1) for h in (heads, heads, heads * group))

    def calls():
        cache = filled(batch, heads, dim, 3)
        sq.squant_cache_write(cache, k, v, *batch.args)
        out = [cache]
        for dtype in (BF16, FP16):
            buffers = [torch.zeros((batch.rows, heads, dim), dtype=dtype, device="cuda") for _ in range(2)]
            sq.squant_cache_read(cache, *batch.args, batch.rows, k=buffers[0], v=buffers[1])
            o = torch.zeros((batch.rows, heads * group, dim), dtype=dtype, device="cuda")
            out += buffers
            for most in {max(news), 0, 1, 2}:
                sq.squant_cache_attention(q.to(dtype), cache, *batch.args, most=most, out=o)
                out.append(o.clone())
        return out

    want = calls()
    sq.use_library(lib_build.LIB_DEBUG)
    try:
        sq.squant_debug_violations()
        got = calls()
        checked, failed, site = sq.squant_debug_violations()
        assert checked and failed == 0, (failed, site)
    finally:
        sq.use_library(None)
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and _status() == 0


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("news,most", [(1, 1), (3, 3), (150, 0)])
def test_calls_that_give_up_end_and_leave_the_gpu_usable(checked_build, dim, news, most):
    """Without a try every wait gives up at once: the call ends, the status says so once, and later calls are right."""
    batch = Batch([900, 300], [news, news], 32)
    cache = filled(batch, 2, dim, 3)
    q = inputs(batch.rows, 8, dim, BF16, 4)
    want = sq.squant_cache_attention(q, cache, *batch.args, most=most)
    assert _status() == 0
    for tries in (0, 1, 0):
        assert sq.squant_debug_linear_wait_limit(tries)
        sq.squant_cache_attention(q, cache, *batch.args, most=most)
        assert _status() in ((-10,) if tries == 0 else (-10, 0))
        assert sq.squant_debug_linear_wait_limit(-1)
        assert torch.equal(sq.squant_cache_attention(q, cache, *batch.args, most=most), want) and _status() == 0
