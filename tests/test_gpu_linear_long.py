"""Contractions longer than one accumulator takes (65,536 terms): the linear operators share them out or take them in parts whose sums are
added in fp32."""
import pytest
import torch

import paper_2202_07471_b200 as sq
from linear_cases import decode64, encode64, gen, int_layer, pack, padded, same_bits

pytestmark = pytest.mark.gpu

LONGEST = 1 << 16


def _sparse(rows, cols, seed, each=10):
    """-1, 0 and 1, one in `each` not zero."""
    v = torch.randint(-each, each + 1, (rows, cols), generator=gen(seed), device="cuda", dtype=torch.int8)
    return torch.where(v.abs() == 1, v, torch.zeros_like(v))


# channels of few_kernel's warps and fused_kernel's thread blocks at their limit of 8 * 65,536 terms, and behind it; parts of dense_kernel
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("tokens,cin,cout,pad,launches", [(1, 8 * LONGEST, 17, 0, 1), (3, 8 * LONGEST + 32, 20, 0, 10), (8, 8 * LONGEST + 32, 20, 0, 10),
                                                          (1, 8 * LONGEST + 3, 9, 0, 10), (40, 8 * LONGEST, 33, 0, 1), (40, 8 * LONGEST + 32, 33, 0, 10),
                                                          (40, LONGEST + 32, 130, 0, 1), (40, 2 * LONGEST + 1, 65, 1, 2), (300, LONGEST, 40, 0, 2),
                                                          (300, LONGEST + 32, 40, 0, 3), (300, LONGEST + 1, 300, 3, 4), (700, 2 * LONGEST + 32, 600, 0, 4)])
def test_forward_of_integers_is_exact(tokens, cin, cout, pad, launches, bits):
    codes, scales = int_layer(cin, cout, bits, 1)
    x, _ = padded(_sparse(tokens, cin, 2).bfloat16(), pad)
    stored = pack(codes) if bits == 4 else codes
    bias = torch.randint(-9, 10, (cout,), generator=gen(3), device="cuda").float()
    res = torch.randint(-20, 21, (tokens, cout), generator=gen(4), device="cuda").bfloat16()
    mass = x.double().abs() @ codes.double().abs().T
    assert mass.max() < 2 ** 24   # sums in any order are exact
    z = (x.double() @ codes.double().T) * scales.double() + bias.double()
    assert (z.float().double() == z).all() and ((z + res.double()).float().double() == z + res.double()).all()
    n = sq.squant_launch_count()
    y = sq.squant_linear(x, stored, scales, bias, residual=res, act="relu", pack_int4=bits == 4)
    assert sq.squant_launch_count() == n + launches
    assert same_bits(y + 0.0, (z.clamp(min=0) + res.double()).to(torch.bfloat16) + 0.0)
    y, z8 = sq.squant_linear(x, stored, scales, bias, pack_int4=bits == 4, checkpoint=True)
    q, e = encode64(z)
    assert same_bits(y + 0.0, z.to(torch.bfloat16) + 0.0) and torch.equal(z8.codes, q) and torch.equal(z8.exps, e)
    sq.squant_device_status()


def test_more_tiles_than_thread_blocks():
    """Every tile would have one thread block for itself, but for its contraction's length."""
    tokens, cin, cout = 40, LONGEST + 64, 40000
    some = torch.randint(-128, 128, (50, cin), generator=gen(1), device="cuda", dtype=torch.int32).to(torch.int8)
    x = _sparse(tokens, cin, 2).bfloat16()
    y = sq.squant_linear(x, some.repeat(cout // 50, 1), torch.ones(cout, device="cuda"))
    assert same_bits(y + 0.0, (x.double() @ some.double().T).to(torch.bfloat16).repeat(1, cout // 50) + 0.0)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("tokens,cin,cout", [(300, 40, LONGEST + 5), (5, 33, 8 * LONGEST + 1), (64, 64, 8 * LONGEST), (LONGEST + 1, 65, 40), (2 * LONGEST + 64, 264, 130)])
def test_gradients_of_integers_are_exact(tokens, cin, cout, bits):
    codes, _ = int_layer(cin, cout, bits, 1)
    scales = torch.full((cout,), 0.5, device="cuda")
    dy = _sparse(tokens, cout, 2).bfloat16()
    x = torch.randint(-5, 6, (tokens, cin), generator=gen(3), device="cuda").bfloat16()
    assert (dy.double().abs() @ codes.double().abs()).max() < 2 ** 24
    g = sq.squant_linear_backward(dy, pack(codes) if bits == 4 else codes, scales, cin=cin, pack_int4=bits == 4, x=sq.squant_checkpoint(x), dweight=True, dbias=True)
    assert same_bits(g.dx + 0.0, (dy.double() @ codes.double() * 0.5).to(torch.bfloat16) + 0.0)
    assert same_bits(g.dweight + 0.0, (dy.double().T @ x.double()).to(torch.bfloat16) + 0.0)
    assert torch.equal(g.dbias.double(), dy.double().sum(0))
    sq.squant_device_status()


# What sums of positive terms may lose: a part has at most 65,536 terms, 4,096 additions of 16 products each, every one of which cuts off less than two
# last places (2^-23) of the sum; parts are added to the nearest, and the result is rounded by half a step.
CUT, HALF = 2 * 4096 * 2.0 ** -23, 2.0 ** -8


def test_sums_of_one_sign_keep_their_value():
    """In one accumulator 2^21 terms lose 1.2 % of their sum."""
    tokens = 1 << 21
    dy = torch.rand((tokens, 64), generator=gen(1), device="cuda").bfloat16()
    x8 = sq.squant_checkpoint(torch.rand((tokens, 64), generator=gen(2), device="cuda").bfloat16())
    n = sq.squant_launch_count()
    got = sq.squant_linear_backward(dy, torch.ones((64, 64), device="cuda", dtype=torch.int8), torch.ones(64, device="cuda"), x=x8, dx=False, dweight=True).dweight
    assert sq.squant_launch_count() == n + 1 + tokens // LONGEST
    want = dy.double().T @ decode64(x8.codes, x8.exps, 64)
    assert ((got.double() - want).abs() <= (HALF + CUT + tokens // LONGEST * 2.0 ** -24) * want).all()
    x = torch.rand((300, 1 << 20), generator=gen(3), device="cuda").bfloat16()
    codes = torch.randint(0, 128, (64, 1 << 20), generator=gen(4), device="cuda", dtype=torch.int32).to(torch.int8)
    want = x.double() @ codes.double().T
    for rows in (x, x[:40], x[:3]):
        y = sq.squant_linear(rows, codes, torch.ones(64, device="cuda"))
        assert ((y.double() - want[:len(rows)]).abs() <= (HALF + CUT + 16 * 2.0 ** -24) * want[:len(rows)]).all()


def test_a_contraction_of_many_parts():
    """2^27 tokens of a layer of one tile: a third of a second."""
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB")
    base, times = 1 << 17, 1 << 10
    dy = torch.randint(0, 4, (base, 32), generator=gen(1), device="cuda").bfloat16()
    x = torch.randint(0, 4, (base, 32), generator=gen(2), device="cuda").bfloat16()
    want = (dy.double().T @ x.double()) * times
    x8 = sq.squant_checkpoint(x)
    x8 = sq.Checkpoint(x8.codes.repeat(times, 1), x8.exps.repeat(times, 1), 32)
    got = sq.squant_linear_backward(dy.repeat(times, 1), torch.ones((32, 32), device="cuda", dtype=torch.int8), torch.ones(32, device="cuda"), x=x8, dx=False,
                                    dweight=True).dweight
    sq.squant_device_status()
    parts = base * times // LONGEST
    assert ((got.double() - want).abs() <= (HALF + CUT + parts * 2.0 ** -24) * want).all()
