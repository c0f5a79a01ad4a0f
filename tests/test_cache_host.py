"""Arguments of the key/value cache's operators: what the library and the binding refuse before any CUDA call (no GPU needed)."""
import ctypes

import pytest
import torch

import paper_2202_07471_b200 as sq
from paper_2202_07471_b200 import binding, cache

OK_PTR, ODD_PTR = 1 << 20, (1 << 20) + 1   # never dereferenced


def rows(**kw):
    r = cache.CacheRows(data=OK_PTR, page_count=10, kv_heads=2, head_dim=128, page_size=64, batch=3, width=4, lens=OK_PTR, pages=OK_PTR, pages_stride=4,
                        starts=OK_PTR, rows=7)
    for k, v in kw.items():
        setattr(r, k, v)
    return r


def move(**kw):
    own = {k: kw.pop(k) for k in list(kw) if k != "rows" and k in dict(cache.CacheMoveArgs._fields_)}
    a = cache.CacheMoveArgs(rows=rows(**kw), dtype=0, k=OK_PTR, v=OK_PTR, k_stride=256, k_head_stride=128, v_stride=256, v_head_stride=128)
    for k, v in own.items():
        setattr(a, k, v)
    return a


def attention(**kw):
    own = {k: kw.pop(k) for k in list(kw) if k != "rows" and k in dict(cache.CacheAttentionArgs._fields_)}
    a = cache.CacheAttentionArgs(rows=rows(**kw), dtype=0, group=4, most=0, scale=0.1, q=OK_PTR, q_stride=1024, q_head_stride=128, out=OK_PTR, out_stride=1024,
                                 out_head_stride=128)
    for k, v in own.items():
        setattr(a, k, v)
    return a


COMMON = [({"head_dim": 96}, -2), ({"head_dim": 0}, -2), ({"page_size": 0}, -2), ({"page_size": 24}, -2), ({"page_size": (1 << 24) + 16}, -2), ({"kv_heads": 0}, -2),
          ({"kv_heads": (1 << 16) + 1}, -2), ({"page_count": -1}, -2), ({"page_count": 1 << 31}, -2), ({"batch": -1}, -2), ({"width": -1}, -2), ({"rows": -1}, -2), ({"rows": (1 << 30) + 1}, -2),
          ({"pages_stride": 3}, -2), ({"starts": None}, -2), ({"dtype": 2}, -4), ({"data": None}, -1), ({"lens": None}, -1), ({"pages": None}, -1), ({"data": OK_PTR + 8}, -5),
          ({"lens": OK_PTR + 2}, -5), ({"pages": OK_PTR + 1}, -5), ({"starts": OK_PTR + 2}, -5)]


@pytest.mark.parametrize("kw,code", COMMON + [({"k": None}, -1), ({"v": None}, -1), ({"k": ODD_PTR}, -5), ({"v": ODD_PTR}, -5), ({"k_stride": -1}, -2), ({"v_head_stride": -128}, -2),
                                              ({"k_stride": (1 << 36) + 1}, -2)])
def test_write_and_read_refuse(kw, code):
    lib = cache._lib()
    assert lib.squant_cache_write(ctypes.byref(move(**kw)), None) == code
    assert lib.squant_cache_read(ctypes.byref(move(**kw)), None) == code


@pytest.mark.parametrize("kw", [{"k_stride": 255}, {"v_head_stride": 127}, {"k_stride": 0}, {"k_stride": 128, "k_head_stride": 128}])
def test_read_refuses_rows_that_lie_in_one_another(kw):
    lib = cache._lib()
    assert lib.squant_cache_read(ctypes.byref(move(**kw)), None) == -2


@pytest.mark.parametrize("kw,code", COMMON + [
    ({"group": 0}, -2), ({"group": (1 << 16) + 1}, -2), ({"group": 1 << 16, "kv_heads": 64}, -2), ({"rows": 1 << 30, "group": 2}, -2), ({"group": 1 << 8, "width": 1 << 20, "pages_stride": 1 << 20, "page_size": 1 << 10, "out_stride": 1 << 20}, -2), ({"most": -1}, -2), ({"q_stride": -1}, -2),
    ({"out_stride": 1023}, -2), ({"out_head_stride": 100}, -2), ({"scale": float("nan")}, -4), ({"scale": float("inf")}, -4), ({"q": None}, -1), ({"out": None}, -1), ({"q": ODD_PTR}, -5),
    ({"out": ODD_PTR}, -5), ({"lse": OK_PTR + 2}, -5), ({}, -12), ({"workspace": OK_PTR, "workspace_bytes": 16}, -12), ({"workspace": OK_PTR + 8, "workspace_bytes": 1 << 40}, -12)])
def test_attention_refuses(kw, code):
    lib = cache._lib()
    a = attention(**kw)
    assert lib.squant_cache_attention(ctypes.byref(a), None) == code
    if code != -12:
        assert lib.squant_cache_attention_workspace(ctypes.byref(a)) == code and lib.squant_cache_attention_plan(ctypes.byref(a)) == code


def test_null_arguments_and_calls_without_rows():
    lib = cache._lib()
    assert lib.squant_cache_write(None, None) == lib.squant_cache_read(None, None) == lib.squant_cache_attention(None, None) == -1
    assert lib.squant_cache_attention_workspace(None) == lib.squant_cache_attention_plan(None) == -1
    for kw in ({"rows": 0}, {"batch": 0}):
        a, m = attention(data=None, lens=None, pages=None, q=None, out=None, **kw), move(data=None, lens=None, pages=None, k=None, v=None, **kw)
        assert lib.squant_cache_attention_workspace(ctypes.byref(a)) == 0 and lib.squant_cache_attention_plan(ctypes.byref(a)) == 0
        assert lib.squant_cache_attention(ctypes.byref(a), None) == 0
        assert lib.squant_cache_write(ctypes.byref(m), None) == 0 and lib.squant_cache_read(ctypes.byref(m), None) == 0


def test_plans():
    """Which kernel: by rows times heads of a group, at most, of a sequence, as far as the host knows."""
    lib = cache._lib()
    plan = lambda **kw: lib.squant_cache_attention_plan(ctypes.byref(attention(**{"out_stride": 1 << 20, **kw})))
    assert plan(starts=None, rows=3) == 1 and plan(starts=None, rows=3, group=40) == 1 and plan(starts=None, rows=3, group=41) == 3
    assert plan() == 1 and plan(rows=11) == 3 and plan(rows=11, most=10) == 1 and plan(rows=11, most=11) == 3
    for dim, most in ((64, 64), (256, 48)):
        assert [plan(head_dim=dim, starts=None, rows=3, group=g, out_head_stride=dim) for g in (8, 9, most, most + 1)] == [1, 2, 2, 3]
    need = lambda **kw: lib.squant_cache_attention_workspace(ctypes.byref(attention(out_stride=1 << 20, out_head_stride=256, **kw)))
    for dim in (64, 128, 256):
        for kw in ({"most": 1}, {"most": 4}, {}):
            small, large = need(head_dim=dim, **kw), need(head_dim=dim, rows=1 << 20, width=1 << 12, pages_stride=1 << 12, **kw)
            assert 0 < small <= large < 1 << 27   # bounded, however much there is to do
    assert need(width=0, most=1) > 0              # rows that see nothing are written too


def test_binding_refuses():
    c = torch.zeros((4, 2, 4, 18 * 64), dtype=torch.uint8)
    lens, pages, starts = torch.zeros(3, dtype=torch.int32), torch.zeros((3, 2), dtype=torch.int32), torch.zeros(4, dtype=torch.int32)
    assert cache._cache_rows(c, lens, pages, starts, 5).page_size == 64
    for bad in ((c.int(), lens, pages, starts), (c[:, :, :, :100], lens, pages, starts), (c.transpose(0, 1), lens, pages, starts), (c, lens.long(), pages, starts),
                (c, lens[None], pages, starts), (c, lens, pages[:2], starts), (c, lens, pages.t().contiguous().t(), starts), (c, lens, pages, starts[:3]), (c, lens, pages, None)):
        with pytest.raises(ValueError):
            cache._cache_rows(*bad, 5)
    x = torch.zeros((5, 2, 64), dtype=torch.bfloat16)
    for bad in (x.float(), x[:4], x[:, :1], x[..., :32], x.transpose(1, 2).contiguous().transpose(1, 2)):
        with pytest.raises(ValueError):
            cache._heads(bad, 5, 2, 64, "k", x.device, None)
    for call in (lambda: sq.squant_cache_write(c, x, x, lens, pages, starts), lambda: sq.squant_cache_read(c, lens, pages, starts, 5),
                 lambda: sq.squant_cache_attention(x, c, lens, pages, starts)):
        with pytest.raises(ValueError, match="CUDA"):
            call()
    with pytest.raises(ValueError, match="autograd"):
        sq.squant_cache_attention(x.requires_grad_(), c, lens, pages, starts)
    for kw in ({"pages": -1}, {"kv_heads": 0}, {"head_dim": 96}, {"page_size": 20}, {"page_size": 0}):
        with pytest.raises(ValueError):
            sq.alloc_cache(**{"pages": 3, "kv_heads": 2, "head_dim": 64, "device": "cpu", **kw})
    assert sq.alloc_cache(3, 2, 64, device="cpu").shape == (3, 2, 4, 1152)


def test_native_arguments_are_the_binding_s():
    if binding._marshal is None:
        pytest.skip("the extension has not been built")
    assert binding._marshal.cache_move_bytes == ctypes.sizeof(cache.CacheMoveArgs) and binding._marshal.cache_attention_bytes == ctypes.sizeof(cache.CacheAttentionArgs)
