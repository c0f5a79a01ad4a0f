"""What the key/value cache's binding and library refuse beyond the common mistakes (no GPU needed)."""
import ctypes

import pytest
import torch
from torch.autograd import forward_ad

import paper_2202_07471_b200 as sq
from paper_2202_07471_b200 import cache
from test_cache_host import attention, move

I32 = torch.int32


def parts(batch=3, width=2):
    return torch.zeros(batch, dtype=I32), torch.zeros((batch, width), dtype=I32), torch.zeros(batch + 1, dtype=I32)


@pytest.mark.parametrize("shape", [(4, 0, 4, 1152), (4, 2, 0, 1152), (0, 0, 0, 1152)])
def test_a_cache_without_heads_or_positions_is_refused(shape):
    with pytest.raises(ValueError, match="cache"):
        cache._cache_rows(torch.zeros(shape, dtype=torch.uint8), *parts(), 5)
    assert cache._cache_rows(torch.zeros((0, 2, 4, 1152), dtype=torch.uint8), *parts(), 5).page_count == 0   # no pages: everything counts as not there


def test_counts_beyond_32_bits_are_refused():
    """The library's descriptor holds them in 32: a count that does not fit must not come out as another one.  (Tensors without storage stand for large ones.)"""
    def rows(shape=(4, 2, 4, 1152), batch=3, width=2):
        empty = lambda *s: torch.empty(s, dtype=I32, device="meta")
        return cache._cache_rows(torch.empty(shape, dtype=torch.uint8, device="meta"), empty(batch), empty(batch, width), empty(batch + 1), 5)

    assert rows().batch == 3 and rows(width=2 ** 31 - 1).width == 2 ** 31 - 1
    for kw in ({"batch": 2 ** 32 + 3}, {"batch": 2 ** 31}, {"width": 2 ** 32 + 2}, {"width": 2 ** 31}, {"shape": (1, 2 ** 32 + 2, 4, 1152)}, {"shape": (1, 2, 2 ** 28 + 4, 1152)}):
        with pytest.raises(ValueError, match="32 bits"):
            rows(**kw)


@pytest.mark.parametrize("kw", [{"page_count": 1 << 31, "kv_heads": 1 << 16, "page_size": 16 << 17}, {"page_count": 1 << 31, "kv_heads": 1 << 14, "page_size": 16 << 19},
                                {"batch": (1 << 30) + 1, "pages_stride": 1 << 3}, {"batch": (1 << 31) - 1}])
def test_products_and_counts_that_overflow_are_refused(kw):
    """Granules are counted with care for 64 bits; the walks over the sequences count in 32, in steps of 32 and by the 32nd part."""
    lib = cache._lib()
    assert lib.squant_cache_write(ctypes.byref(move(k_stride=1 << 30, v_stride=1 << 30, **kw)), None) == -2
    assert lib.squant_cache_read(ctypes.byref(move(k_stride=1 << 30, v_stride=1 << 30, **kw)), None) == -2
    assert lib.squant_cache_attention_plan(ctypes.byref(attention(out_stride=1 << 30, group=1, **kw))) == -2


def test_rows_in_one_another_are_refused_where_their_distance_overflows():
    """(rows - 1) strides beyond 64 bits: heads on top of one another, not heads apart by all the rows."""
    lib = cache._lib()
    for rows, stride, head in ((1 << 28, 1 << 36, 0), (1 << 28, 1 << 36, 127), (1 << 30, 1 << 34, 64)):
        assert lib.squant_cache_attention_plan(ctypes.byref(attention(rows=rows, group=1, out_stride=stride, out_head_stride=head))) == -2
        assert lib.squant_cache_read(ctypes.byref(move(rows=rows, k_stride=stride, k_head_stride=head)), None) == -2
        assert lib.squant_cache_read(ctypes.byref(move(rows=rows, v_stride=stride, v_head_stride=head)), None) == -2
    # heads apart by all the rows, and rows apart by all the heads
    for stride, head in ((128, 7 * 128), (256, 128), (130, 6 * 130 + 128), (3 * 128, 128)):
        assert lib.squant_cache_attention_plan(ctypes.byref(attention(group=1, out_stride=stride, out_head_stride=head))) > 0
    for stride, head in ((128, 7 * 128 - 1), (255, 128), (130, 6 * 130 + 127), (256, 127), (0, 128)):
        assert lib.squant_cache_attention_plan(ctypes.byref(attention(group=1, out_stride=stride, out_head_stride=head))) == -2


def test_scales_beyond_fp32_are_refused():
    lib = cache._lib()
    for scale, code in ((3e38, -4), (-3.4e38, -4), (2.3e38, 1), (0.0, 1), (-1e-45, 1)):
        assert lib.squant_cache_attention_plan(ctypes.byref(attention(scale=scale))) == code


def test_tangents_are_refused():
    """A forward-mode derivative would be lost without a word, whatever grad mode is."""
    c, x, (lens, pages, starts) = torch.zeros((4, 2, 4, 18 * 64), dtype=torch.uint8), torch.zeros((5, 2, 64), dtype=torch.bfloat16), parts()
    with forward_ad.dual_level(), torch.no_grad():
        dual = forward_ad.make_dual(x, x)
        for call in (lambda: sq.squant_cache_attention(dual, c, lens, pages, starts), lambda: sq.squant_cache_write(c, dual, x, lens, pages, starts),
                     lambda: sq.squant_cache_write(c, x, dual, lens, pages, starts), lambda: sq.squant_cache_attention(x, c, lens, pages, starts, out=dual)):
            with pytest.raises(ValueError, match="tangent"):
                call()
        with pytest.raises(ValueError, match="CUDA"):
            sq.squant_cache_attention(x, c, lens, pages, starts)
