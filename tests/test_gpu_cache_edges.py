"""The key/value cache at its edges: scores that grow inside what is taken at once, calls that repeat, captured calls that have given up, fp16 at both ends."""
import ctypes

import pytest
import torch
from torch.autograd import forward_ad

import paper_2202_07471_b200 as sq
from cache_cases import Batch, attention, filled, gen, pack, stored
from paper_2202_07471_b200 import build as lib_build, cache as cache_module
from test_gpu_cache import BF16, FP16, check_attention, inputs, same

pytestmark = pytest.mark.gpu
PROMPT = 3


def plan(q, cache, batch, most):
    """Which kernel a call takes."""
    a = cache_module.CacheAttentionArgs(cache_module._cache_rows(cache, *batch.args, q.shape[0]), 0, q.shape[1] // cache.shape[1], most, 1.0, q.data_ptr(),
                                        q.stride(0), q.stride(1), q.data_ptr(), q.shape[1] * q.shape[2], q.shape[2])
    return cache_module._lib().squant_cache_attention_plan(ctypes.byref(a))


def rising(batch, heads, dim, levels, v_scale=1.0):
    """A cache whose position p has the score levels[p], in powers of two, for a query of ones: keys of one magnitude, which the codes keep to 2^-5."""
    v = torch.randn((batch.page_count, heads, batch.page_size // 16, 16, dim), generator=gen(2), device="cuda") * v_scale
    k = torch.zeros_like(v)
    for b, n in enumerate(batch.lens_list):
        for p in range(n):
            k[batch.pages_list[b, p // batch.page_size], :, p % batch.page_size // 16, p % 16] = levels[p] / dim
    return pack(k.to(BF16), v.to(BF16))


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("news", [[300, 170], [20, 9], [16, 9]])
@pytest.mark.parametrize("jumps", [(13, 2), (2, 13), (9, 15), (15, 15, 15), (0, 14, 0, 3, 15, 13), (13, 13, 2, 2)])
def test_scores_that_grow_several_times_in_one_tile(dim, dtype, news, jumps):
    """A row whose maximum is replaced inside a score tile has what is there scaled while it is being made: its weights, and its sums, which may just have been scaled for the
    tile before.  Every 32 positions, which are taken together, the scores rise by another jump, less or more than a weight's type has room for (2^14 in fp16,
    2^64 in bf16); what came before the jump keeps a part in the result, and would be far too large if it were scaled too little."""
    heads, group = 2, 8
    room = 1.0 if dtype == FP16 else 64.0 / 14
    batch = Batch([300, 170], news, 16, seed=5)
    level, levels = 0.0, []
    for i in range(-(-300 // 32)):
        level += jumps[i % len(jumps)] * room if i >= 2 else 0
        levels += [level] * 32
    cache = rising(batch, heads, dim, levels)
    q = (1 + 0.02 * torch.randn((batch.rows, heads * group, dim), generator=gen(7), device="cuda")).to(dtype)
    assert plan(q, cache, batch, max(news)) == PROMPT
    scale = 0.6931471805599453
    out, lse = sq.squant_cache_attention(q, cache, *batch.args, most=max(news), lse=True, scale=scale)
    # a weight is rounded once: it is scaled by powers of two
    check_attention(out, lse, q, batch, cache, scale, rounded_p=max(news) * group > 128)
    again, lse_again = sq.squant_cache_attention(q, cache, *batch.args, most=max(news), lse=True, scale=scale)
    assert torch.equal(out, again) and torch.equal(lse, lse_again)
    assert sq.squant_device_status() is None


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("group,news", [(4, 1), (12, 1), (5, 3)])
def test_steps_repeat_to_the_bit(dim, group, news):
    """A place in shared memory is given back to the copies behind the loads from it: many short pages, so that copies are small and quick, and every call the same."""
    batch = Batch([4000, 33, 700, 2049] * 8, [news] * 32, 16, seed=6)
    cache = filled(batch, 2, dim, 3)
    for dtype in (BF16, FP16):
        q = inputs(batch.rows, 2 * group, dim, dtype, 4)
        want = sq.squant_cache_attention(q, cache, *batch.args, most=news)
        for _ in range(60):
            assert torch.equal(sq.squant_cache_attention(q, cache, *batch.args, most=news), want)
    assert sq.squant_device_status() is None


@pytest.fixture
def checked_build():
    sq.use_library(lib_build.LIB_DEBUG)
    try:
        yield
    finally:
        sq.squant_debug_linear_wait_limit(-1)
        sq.use_library(None)


def status():
    try:
        sq.squant_device_status()
        return 0
    except sq.SquantError as e:
        return e.code


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("news,most", [(1, 1), (150, 0)])
def test_a_captured_call_is_right_again_after_it_has_given_up(checked_build, dim, news, most):
    """Waits of one to six tries run out in some blocks and not in others: those that share a tile have counted, and a replay, whose number is the same, starts from no count."""
    batch = Batch([900, 300, 520], [news] * 3, 32)
    cache = filled(batch, 2, dim, 3)
    q = inputs(batch.rows, 8, dim, BF16, 4)
    out = torch.empty(q.shape, dtype=BF16, device="cuda")
    want = sq.squant_cache_attention(q, cache, *batch.args, most=most)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sq.squant_cache_attention(q, cache, *batch.args, most=most, out=out)
    assert status() == 0
    gave_up = 0
    for tries in (1, 2, 3, 4, 6) * 6 + (0,):
        assert sq.squant_debug_linear_wait_limit(tries)
        graph.replay()
        gave_up += status() == -10
        assert sq.squant_debug_linear_wait_limit(-1)
        for _ in range(2):
            out.zero_()
            graph.replay()
            assert torch.equal(out, want) and status() == 0, tries
    assert gave_up > 0


def magnitudes(dim):
    """Rows of every power of two from 2^-40 on, with the mantissas 1, 9/8, 5/4 and 15/8 of a group's largest value and codes of every size; groups of zeros, of values that are too small and without a number."""
    rows = []
    for exponent in range(-40, 121):
        tops = torch.tensor([1.0, 1.125, 1.25, 1.875], dtype=torch.float64).repeat(dim // 128 + 1)[:dim // 32] * 2.0 ** exponent
        parts = torch.linspace(-1, 1, 32, dtype=torch.float64)
        rows.append((tops[:, None] * parts).flatten())
    special = torch.ones(dim, dtype=torch.float64)
    special[:32], special[32] = 0.0, float("nan")
    rows.append(special)
    rows.append(torch.full((dim,), 2.0 ** -101, dtype=torch.float64))
    return torch.stack(rows)[:, None, :].to(BF16).cuda()


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_fp16_values_are_rounded_once_at_every_magnitude(dim):
    """code * scale, rounded to nearest: also where fp16 holds the values and not the scale, and zeros where the scale is beyond fp16."""
    k = magnitudes(dim)
    v = k.flip(0).contiguous()
    n = k.shape[0]
    batch = Batch([n], [n], 32)
    cache = sq.alloc_cache(batch.page_count, 1, dim, page_size=32)
    sq.squant_cache_write(cache, k, v, *batch.args)
    rk, rv = sq.squant_cache_read(cache, *batch.args, n, dtype=FP16)
    for got, x in ((rk, k), (rv, v)):
        want = stored(x).float().half()   # a value has seven bits: exact in fp32
        assert want.isinf().any() and (want == 2.0 ** -24).any() and (want == 0).any() and same(got, want)
    slices = torch.empty((n, 1, dim + 3), dtype=FP16, device="cuda"), torch.empty((n, 1, dim + 3), dtype=FP16, device="cuda")
    sq.squant_cache_read(cache, *batch.args, n, k=slices[0][..., 3:], v=slices[1][..., 3:])
    assert same(slices[0][..., 3:], rk) and same(slices[1][..., 3:], rv)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("news", [1, 2, 40])
def test_fp16_attention_to_small_and_large_values(dim, news):
    """Of the sizes that fp16 holds: exact values from 2^-18 up to 65,504 (a group's largest); below, the scale is rounded to a multiple of 2^-24, by half of one, and so is
    its product with the code: up to 7 * 2^-25 + 2^-25 = 2^-22 off, and so is a value's average."""
    heads, group, n = 1, 8, 48
    batch = Batch([n], [news], 16)
    for top, off in ((65504.0, 0.0), (2.0 ** -18, 0.0), (2.0 ** -21, 2.0 ** -22), (5 * 2.0 ** -24, 2.0 ** -22), (2.0 ** -24, 2.0 ** -22)):
        k = torch.zeros((n, heads, dim), dtype=FP16, device="cuda")
        v = (torch.rand((n, heads, dim), generator=gen(1), device="cuda") * 2 - 1) * top
        v[..., ::32] = top
        cache = sq.alloc_cache(batch.page_count, heads, dim, page_size=16)
        every = Batch([n], [n], 16)
        sq.squant_cache_write(cache, k, v.to(FP16), every.lens, batch.pages, every.starts)
        q = inputs(news, heads * group, dim, FP16, 3)
        out = sq.squant_cache_attention(q, cache, *batch.args, most=news)
        want, _ = attention(q, batch, cache)
        size = stored(v.to(FP16)).abs().amax()
        # what the kernels round besides (see check_attention), a weight at most 2^-11 and 2^-25
        assert ((out.double() - want).abs() <= off + 2.0 ** -11 * want.abs() + 2.0 ** -25 + (2.0 ** -11 + 2.0 ** -16 + n * 2.0 ** -25) * size).all(), top
        assert top < 1e-5 or not out.isnan().any() and (out != 0).any()


def test_a_cache_without_heads_or_positions_is_refused():
    """By every call, with the binding's error: the native calls divide by the number of heads."""
    batch = Batch([4, 1], [1, 1], 16)
    for shape in ((4, 0, 4, 1152), (4, 2, 0, 1152)):
        cache = torch.zeros(shape, dtype=torch.uint8, device="cuda")
        x = inputs(2, 2, 64, BF16, 1)
        for call in (lambda: sq.squant_cache_write(cache, x[:, :shape[1]], x[:, :shape[1]], *batch.args), lambda: sq.squant_cache_read(cache, *batch.args, 2),
                     lambda: sq.squant_cache_attention(x, cache, *batch.args)):
            with pytest.raises(ValueError):
                call()


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("group,lens,news", [(4, [300, 33, 1, 0, 700], [1, 1, 1, 0, 1]), (8, [260, 64, 1000], [16, 3, 9]), (16, [129, 500], [8, 1]), (1, [700, 128, 90], [128, 100, 90]),
                                             (5, [1300, 40], [8, 8])])
def test_short_sequences_keep_all_of_their_weights(dim, dtype, group, lens, news):
    """Sequences of up to 128 rows (tokens times query heads of a kv head) come to any kernel, by what is known of the others: weights lose nothing in any of them, so results differ
    in the last places alone."""
    batch = Batch(lens, news, 32, seed=3)
    cache = filled(batch, 2, dim, 5)
    q = inputs(batch.rows, 2 * group, dim, dtype, 3)
    plans = set()
    for most in (0, max(news), 1):
        plans.add(plan(q, cache, batch, most))
        out, lse = sq.squant_cache_attention(q, cache, *batch.args, most=most, lse=True)
        check_attention(out, lse, q, batch, cache, rounded_p=False)
    assert len(plans) > 1 or sum(news) * group <= 40
    assert sq.squant_device_status() is None


def test_a_step_s_precision_does_not_depend_on_the_other_sequences():
    """One token of each sequence, with starts and without a word of how many there are at most: the errors of the output are those of its rounding."""
    batch = Batch([600 + 7 * i for i in range(24)], [1] * 24, 64)
    cache = filled(batch, 4, 128, 5)
    q = inputs(24, 16, 128, BF16, 3)
    want, _ = attention(q, batch, cache)
    errors = []
    for most in (1, 0):
        out = sq.squant_cache_attention(q, cache, *batch.args, most=most)
        errors.append(float(torch.linalg.norm(out.double() - want) / torch.linalg.norm(want)))
    rounded = float(torch.linalg.norm(want.to(BF16).double() - want) / torch.linalg.norm(want))
    assert plan(q, cache, batch, 0) == PROMPT and max(errors) <= 1.01 * rounded, (errors, rounded)


def test_tangents_are_refused():
    """By the native calls too; what a tangent has been taken off is an ordinary tensor again."""
    batch = Batch([40, 17], [3, 1], 16)
    cache = filled(batch, 2, 64, 3)
    q, k = inputs(4, 8, 64, BF16, 4), inputs(4, 2, 64, BF16, 5)
    want = sq.squant_cache_attention(q, cache, *batch.args)
    with forward_ad.dual_level(), torch.no_grad():
        dq, dk = forward_ad.make_dual(q, q), forward_ad.make_dual(k, k)
        for call in (lambda: sq.squant_cache_attention(dq, cache, *batch.args), lambda: sq.squant_cache_write(cache, dk, k, *batch.args), lambda: sq.squant_cache_write(cache, k, dk, *batch.args),
                     lambda: sq.squant_cache_attention(q, cache, *batch.args, out=dq), lambda: sq.squant_cache_read(cache, *batch.args, 4, k=k, v=dk)):
            with pytest.raises(ValueError, match="tangent"):
                call()
        assert torch.equal(sq.squant_cache_attention(forward_ad.unpack_dual(dq).primal, cache, *batch.args), want)
    assert torch.equal(sq.squant_cache_attention(dq, cache, *batch.args), want)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("news,most", [(300, 0), (20, 0), (3, 3)])
@pytest.mark.parametrize("jumps", [(0, 60), (60, 0), (3, 40, 20)])
def test_large_values_where_scores_grow(dim, news, most, jumps):
    """Values of 2^80: a weight that reaches far beyond the maximum that it is taken against must not carry its product with them out of fp32."""
    batch = Batch([300], [news], 16, seed=5)
    level, levels = 0.0, []
    for i in range(-(-300 // 32)):
        level += jumps[i % len(jumps)] if i >= 3 else 0
        levels += [level] * 32
    cache = rising(batch, 2, dim, levels, v_scale=2.0 ** 80)
    q = (1 + 0.02 * torch.randn((news, 8, dim), generator=gen(7), device="cuda")).to(BF16)
    out, lse = sq.squant_cache_attention(q, cache, *batch.args, most=most, lse=True, scale=0.6931471805599453)
    assert out.isfinite().all()
    check_attention(out, lse, q, batch, cache, 0.6931471805599453, rounded_p=news * 4 > 128)


@pytest.mark.parametrize("news,most", [(100, 0), (20, 0), (1, 1)])
@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_every_finite_scale(dtype, news, most):
    """0: every position counts the same; small ones of large scores are not taken for larger ones; one whose exponents' scale is beyond fp32 is refused."""
    batch = Batch([200, 130], [news, news], 16)
    cache = filled(batch, 2, 64, 5)
    q = inputs(batch.rows, 8, 64, dtype, 3)
    for scale in (0.0, -0.0, 1e-20, 1e-38, 1e-45):
        out, lse = sq.squant_cache_attention(q, cache, *batch.args, most=most, lse=True, scale=scale)
        check_attention(out, lse, q, batch, cache, scale, rounded_p=news * 4 > 128)
    if dtype == BF16:
        shape = (batch.page_count, 2, 1, 16, 64)
        large = pack((torch.randn(shape, generator=gen(1), device="cuda") * 1e17).to(BF16), torch.randn(shape, generator=gen(2), device="cuda").to(BF16))
        far = (q.float() * 1e17).to(BF16)
        for scale in (1e-34, -1e-34, 1e-33):
            out, lse = sq.squant_cache_attention(far, large, *batch.args, most=most, lse=True, scale=scale)
            check_attention(out, lse, far, batch, large, scale, rounded_p=news * 4 > 128)
    for scale in (3e38, -3.4e38):
        with pytest.raises(sq.SquantError):
            sq.squant_cache_attention(q, cache, *batch.args, most=most, scale=scale)
