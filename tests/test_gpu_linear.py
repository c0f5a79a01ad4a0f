"""The linear operators on the GPU against plain references in 64 bits.

Where x, the codes and the scales are small integers and powers of two, every product, sum and epilogue value is exact in
fp32 and the only rounding is the output's: those tests compare bits.  The others use bounds derived beside them.
"""
import itertools

import pytest
import torch

import paper_2202_07471_b200 as sq
from linear_cases import (ACTS, act64, decode64, encode64, gen, int_layer, pack, padded, real_layer, same_bits, slope64)

pytestmark = pytest.mark.gpu

# either side of every line: the token tiles of the kernel for few tokens (8, 16, 32), one and more row tiles (128),
# contraction stages (64), column tiles (64, 128, 256), rows that start on 16 bytes or not
SHAPES = [(1, 1, 1), (1, 64, 32), (3, 33, 5), (7, 128, 96), (8, 256, 64), (9, 100, 33), (16, 1000, 257), (17, 64, 64), (31, 96, 31), (32, 512, 129),
          (33, 64, 64), (33, 1, 1), (40, 63, 300), (64, 65, 63), (127, 160, 250), (128, 64, 256), (129, 256, 255), (150, 1537, 65),
          (200, 31, 1001), (257, 320, 384), (1, 4096, 512), (300, 128, 8200),
          (40, 4096, 70), (128, 2050, 130), (100, 3000, 64), (20, 4096, 1100), (2, 4090, 40), (2500, 72, 2100), (400, 2100, 300)]


def _ints(shape, lo, hi, seed, dtype):
    return torch.randint(lo, hi + 1, shape, generator=gen(seed), device="cuda").to(dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("tokens,cin,cout", SHAPES)
def test_forward_of_integers_is_exact(tokens, cin, cout, bits, dtype):
    codes, scales = int_layer(cin, cout, bits, 1)
    # |u| <= 3 * 128 * 4096 < 2^24: fp32 sums in any order are exact; fp16: kept inside its range by the scales
    x = _ints((tokens, cin), -3, 3, 2, dtype)
    if dtype == torch.float16:
        scales = scales * 2.0 ** -9
    bias = _ints((cout,), -9, 9, 3, torch.float32)
    res = _ints((tokens, cout), -20, 20, 4, dtype)
    stored = pack(codes) if bits == 4 else codes
    for pad, b, r in ((0, None, None), (0, bias, res), (1, bias, None), (8, None, res)):
        xs, _ = padded(x, pad)
        rs = None if r is None else padded(r, pad)[0]
        y, buf = padded(torch.zeros((tokens, cout), dtype=dtype, device="cuda"), pad, fill=7.0)
        y.fill_(float("nan"))
        got = sq.squant_linear(xs, stored, scales, b, residual=rs, pack_int4=bits == 4, out=y)
        assert got is y
        u = x.double() @ codes.double().T
        z = u * scales.double() + (0 if b is None else b.double())
        assert (z.float().double() == z).all()   # what the comparison to the bit rests on
        want = (z + (0 if r is None else r.double())).to(dtype)
        assert same_bits(y, want), (pad, b is not None, r is not None, (y - want).abs().max())
        assert (buf[:, cout:] == 7.0).all()
    sq.squant_device_status()


# few tokens: rows of x on 32, 16 or fewer bytes, tiles of tokens that end inside, channels that end inside a group of 16; either side
# of the lines between the kernels (50 million codes for 16 tokens, 25 for 32, 8 for 64, 2 for 256)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("tokens", [1, 3, 8, 9, 15, 16, 17, 24, 25, 32, 33, 64, 71, 256])
@pytest.mark.parametrize("cin,cout", [(32, 16), (96, 17), (1056, 40), (2080, 9), (16, 8), (24, 33)])
def test_few_tokens(tokens, cin, cout, bits, dtype):
    codes, scales = int_layer(cin, cout, bits, 1)
    if dtype == torch.float16:
        scales = scales * 2.0 ** -9
    bias, res = _ints((cout,), -9, 9, 3, torch.float32), _ints((tokens, cout), -20, 20, 4, dtype)
    x = _ints((tokens, cin), -3, 3, 2, dtype)
    want = ((x.double() @ codes.double().T) * scales.double() + bias.double() + res.double()).to(dtype)
    for pad, offset in ((0, 0), (16, 0), (8, 0), (16, 8), (32, 16), (1, 0)):
        buf = torch.full((tokens * (cin + pad) + offset + 16,), float("nan"), device="cuda", dtype=dtype)
        xs = buf.as_strided((tokens, cin), (cin + pad, 1), offset)
        xs.copy_(x)
        out = torch.full((tokens + 1, cout + 1), 7.0, device="cuda", dtype=dtype)
        sq.squant_linear(xs, pack(codes) if bits == 4 else codes, scales, bias, residual=res, pack_int4=bits == 4, out=out[:tokens, :cout])
        assert same_bits(out[:tokens, :cout], want), (pad, offset)
        assert (out[tokens:] == 7).all() and (out[:, cout:] == 7).all()


@pytest.mark.parametrize("tokens,cin,cout", [(16, 4096, 12288), (16, 4096, 12304), (32, 4096, 6144), (32, 4096, 6160),
                                             (64, 4096, 2048), (64, 4096, 2064), (65, 1024, 5472), (256, 512, 1024), (256, 512, 1040), (64, 4112, 64)])
def test_either_side_of_the_line_for_few_tokens(tokens, cin, cout):
    codes, scales = int_layer(cin, cout, 4, 1)
    x = _ints((tokens, cin), -3, 3, 2, torch.bfloat16)
    got = sq.squant_linear(x, pack(codes), scales, pack_int4=True)
    assert same_bits(got, ((x.double() @ codes.double().T) * scales.double()).to(torch.bfloat16))
    sq.squant_device_status()


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("bits,dtype,tokens", [(4, torch.bfloat16, 5), (8, torch.float16, 20), (4, torch.float16, 70), (8, torch.bfloat16, 140)])
def test_forward_of_activations(act, bits, dtype, tokens):
    """|y - exact| <= half a step of the output (eps / 2 relative; fp16's smallest step is 2^-24) and what z's error makes of it:
    z is off by at most cin * 2^-23 of the sum of the products' magnitudes (each of cin additions, truncated or rounded, at
    most one last place of partial sums below that), two roundings of the epilogue and, with slopes of at most 1.13, the
    activation's own few last places (16 * 2^-23 of |z|, and of its largest intermediate)."""
    cin, cout = 288, 200
    codes, scales = real_layer(cin, cout, bits, 5)
    x = torch.randn((tokens, cin), generator=gen(6), device="cuda").to(dtype)
    bias = torch.randn((cout,), generator=gen(7), device="cuda")
    res = torch.randn((tokens, cout), generator=gen(8), device="cuda").to(dtype)
    y = sq.squant_linear(x, pack(codes) if bits == 4 else codes, scales, bias, residual=res, act=act, pack_int4=bits == 4)
    s = scales.double()
    z = (x.double() @ codes.double().T) * s + bias.double()
    exact = act64(z, act) + res.double()
    mass = (x.double().abs() @ codes.double().abs().T) * s + bias.double().abs()
    z_off = (cin + 2) * 2.0 ** -23 * mass
    off = 1.13 * z_off + 16 * 2.0 ** -23 * (z.abs() + res.double().abs())
    half = torch.finfo(dtype).eps / 2
    bound = off + half * (exact.abs() + off) + (2.0 ** -25 if dtype == torch.float16 else 0)
    assert ((y.double() - exact).abs() <= bound).all(), ((y.double() - exact).abs() / bound).max()


@pytest.mark.parametrize("tokens,cin,cout", [(1, 64, 32), (5, 100, 33), (32, 256, 100), (33, 128, 64), (130, 72, 257), (64, 64, 1001)])
def test_forward_saves_its_preactivation(tokens, cin, cout):
    codes, scales = int_layer(cin, cout, 8, 11)
    x = _ints((tokens, cin), -3, 3, 12, torch.bfloat16)
    bias = _ints((cout,), -9, 9, 13, torch.float32)
    y, z = sq.squant_linear(x, codes, scales, bias, act="relu", checkpoint=True)
    exact = (x.double() @ codes.double().T) * scales.double() + bias.double()
    q, e = encode64(exact)
    assert torch.equal(z.exps, e) and torch.equal(z.codes, q)
    assert same_bits(y, exact.clamp(min=0).to(torch.bfloat16) + 0.0)


CHECKPOINT_SHAPES = [(1, 1), (1, 32), (2, 31), (3, 33), (5, 64), (7, 100), (129, 1001), (33, 4096), (1000, 40)]


@pytest.mark.parametrize("rows,features", CHECKPOINT_SHAPES)
@pytest.mark.parametrize("pad", [0, 1, 8])
def test_checkpoint_and_restore(rows, features, pad):
    g = gen(rows * 10007 + features)
    v = torch.randn((rows, features), generator=g, device="cuda") * torch.exp2(torch.randint(-130, 120, (rows, 1), generator=g, device="cuda").float())
    v = torch.where(torch.rand((rows, features), generator=g, device="cuda") < 0.1, torch.zeros_like(v), v)
    x, _ = padded(v.to(torch.bfloat16), pad)
    c = sq.squant_checkpoint(x)
    q, e = encode64(x)
    assert torch.equal(c.codes, q) and torch.equal(c.exps, e)
    back = sq.squant_checkpoint_restore(c)
    want = decode64(q, e, features)
    assert torch.equal(back.double(), want)
    # half a step, a step being 2^(E - 127)
    step = torch.exp2(e.double() - 127).repeat_interleave(32, 1)[:, :features]
    assert ((want - x.double()).abs() <= step / 2).all()


def test_checkpoint_of_special_values():
    inf, nan = float("inf"), float("nan")
    big = torch.finfo(torch.bfloat16).max
    rows = [[0.0] * 32, [-0.0] * 32, [big] + [1.0] * 31, [-big] * 32, [2.0 ** -126] * 32, [2.0 ** -133] * 32, [2.0 ** -133, 2.0 ** -120] * 16,
            [127.0, 0.5, 1.5, 2.5, -0.5, -1.5, 126.5, -126.5] * 4, [127.5, -127.5, 1.0, 0.0] * 8]
    x = torch.tensor(rows, device="cuda").to(torch.bfloat16)
    c = sq.squant_checkpoint(x)
    q, e = encode64(x)
    assert torch.equal(c.codes, q) and torch.equal(c.exps, e)
    bad = torch.ones((4, 70), device="cuda", dtype=torch.bfloat16)
    bad[0, 3], bad[1, 40], bad[2, 69] = inf, nan, -inf
    c = sq.squant_checkpoint(bad)
    got = sq.squant_checkpoint_restore(c)
    poisoned = torch.zeros((4, 70), dtype=torch.bool, device="cuda")
    poisoned[0, :32], poisoned[1, 32:64], poisoned[2, 64:] = True, True, True
    assert torch.equal(torch.isnan(got), poisoned) and (got[~poisoned] == 1).all()
    assert (c.exps == 255).sum() == 3 and (c.codes[0, :32] == 0).all()


def _grads(tokens, cin, cout, bits, act, seed, pad=0, real=True):
    g = gen(seed)
    codes, scales = real_layer(cin, cout, bits, seed) if real else int_layer(cin, cout, bits, seed, -3 if cout > 1000 else -6)
    if real:
        dy = torch.randn((tokens, cout), generator=g, device="cuda").to(torch.bfloat16)
        xv = torch.randn((tokens, cin), generator=g, device="cuda")
        zv = torch.randn((tokens, cout), generator=g, device="cuda")
        bias = torch.randn((cout,), generator=g, device="cuda")
    else:
        dy = _ints((tokens, cout), -2, 2, seed + 1, torch.bfloat16)
        xv = _ints((tokens, cin), -5, 5, seed + 2, torch.float32)
        zv = _ints((tokens, cout), -60, 60, seed + 3, torch.float32)
        bias = _ints((cout,), -3, 3, seed + 4, torch.float32)
    x8, z8 = encode64(xv), encode64(zv)
    return codes, scales, padded(dy, pad)[0], bias, sq.Checkpoint(*x8, cin), sq.Checkpoint(*z8, cout), decode64(*x8, cin), decode64(*z8, cout)


GRAD_SHAPES = [(1, 1, 1), (1, 32, 32), (2, 33, 65), (31, 64, 64), (64, 100, 40), (65, 31, 129), (128, 256, 128), (130, 257, 63), (333, 128, 200), (70, 1001, 37),
               (513, 72, 264), (40, 512, 300), (96, 8200, 32), (50, 65, 2100), (100, 130, 4096), (1000, 300, 2100), (2100, 520, 264)]


@pytest.mark.parametrize("act", ["none", "relu"])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("tokens,cin,cout", GRAD_SHAPES)
def test_gradients_of_integers_are_exact(tokens, cin, cout, bits, act):
    """dy, zhat, xhat, codes and bias are small integers, scales powers of two (2^-6 .. 2^2, from 2^-3 on for many channels): dz * s
    is exact in bf16, and every sum of any of the terms stays below 2^24 of its unit: dx's by the assertion, dweight's are below
    2 * 5 * 2100, dscales' integers below 2 * 63 * 2100."""
    for pad in (0, 1):
        codes, scales, dy, bias, x8, z8, xv, zv = _grads(tokens, cin, cout, bits, act, 21, pad, real=False)
        g = sq.squant_linear_backward(dy, pack(codes) if bits == 4 else codes, scales, bias, cin=cin, act=act, pack_int4=bits == 4, z=z8, x=x8,
                                      dx=True, dweight=True, dbias=True, dscales=True)
        dz = dy.double() * slope64(zv, act)
        assert ((dz.abs() * scales.double()) @ codes.double().abs()).max() * 2.0 ** (3 if cout > 1000 else 6) < 2 ** 24
        assert same_bits(g.dx, ((dz * scales.double()) @ codes.double()).to(torch.bfloat16) + 0.0)
        assert same_bits(g.dweight, (dz.T @ xv).to(torch.bfloat16) + 0.0)
        assert torch.equal(g.dbias.double(), dz.sum(0))
        assert torch.equal(g.dscales.double(), (dz * (zv - bias.double())).sum(0) / scales.double())
    sq.squant_device_status()


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("tokens,cin,cout,bits", [(50, 96, 130, 8), (200, 257, 64, 4)])
def test_gradients_of_real_values(tokens, cin, cout, bits, act):
    """dz and dz * s are rounded to bf16 (2^-9 of each term, 2^-8 counted here: the product dz is itself a few fp32 places
    off), the sums are fp32 and the result is rounded to bf16 (2^-9 of it, 2^-8 counted)."""
    codes, scales, dy, bias, x8, z8, xv, zv = _grads(tokens, cin, cout, bits, act, 31)
    g = sq.squant_linear_backward(dy, pack(codes) if bits == 4 else codes, scales, bias, cin=cin, act=act, pack_int4=bits == 4, z=z8, x=x8,
                                  dx=True, dweight=True, dbias=True, dscales=True)
    slope = slope64(zv, act)
    dz = dy.double() * slope
    # fp32 slope: sums of terms of at most 1 + |z| / sqrt(2 pi), each a few last places off
    dz_off = dy.double().abs() * 16 * 2.0 ** -23 * (1 + zv.abs())
    s, c = scales.double(), codes.double()
    half = 2.0 ** -8
    exact = (dz * s) @ c
    off = ((half * dz.abs() + dz_off) * s + (cout + 2) * 2.0 ** -23 * dz.abs() * s) @ c.abs()
    assert ((g.dx.double() - exact).abs() <= off + half * (exact.abs() + off)).all()
    exact = dz.T @ xv
    off = ((half + (tokens + 2) * 2.0 ** -23) * dz.abs() + dz_off).T @ xv.abs()
    assert ((g.dweight.double() - exact).abs() <= off + half * (exact.abs() + off)).all()
    place = (tokens + 4) * 2.0 ** -24
    exact = dz.sum(0)
    assert ((g.dbias.double() - exact).abs() <= (dz.abs() * place + dz_off).sum(0)).all()
    d = zv - bias.double()
    exact = (dz * d).sum(0) / s
    assert ((g.dscales.double() - exact).abs() <= ((dz.abs() * place * 2 + dz_off) * (d.abs() + bias.double().abs() * 2.0 ** -23)).sum(0) / s).all()


@pytest.mark.parametrize("act", ["gelu", "silu"])
def test_slopes_of_long_columns(act):
    """Codes are the unit matrix and scales 1, so that dx is dz rounded to bf16.  Groups have exponents of all kinds, and the call on all tokens
    gives what calls on a hundred at a time give."""
    tokens, width = 1300, 4096
    codes, scales = torch.eye(width, device="cuda").to(torch.int8), torch.ones(width, device="cuda")
    g = gen(1)
    unit = torch.exp2(torch.randint(-12, 12, (tokens, width // 32), generator=g, device="cuda").float()).repeat_interleave(32, 1)
    z = (torch.randn((tokens, width), generator=g, device="cuda") * unit).to(torch.bfloat16)
    z[7, 100] = float("nan")
    dy = torch.randn((tokens, width), generator=g, device="cuda").to(torch.bfloat16)
    z8 = sq.squant_checkpoint(z)
    got = sq.squant_linear_backward(dy, codes, scales, act=act, z=z8, dbias=True, dscales=True)
    for t in range(0, tokens, 100):
        part = sq.Checkpoint(z8.codes[t:t + 100].clone(), z8.exps[t:t + 100].clone(), width)
        assert same_bits(sq.squant_linear_backward(dy[t:t + 100], codes, scales, act=act, z=part).dx, got.dx[t:t + 100])
    zv = decode64(z8.codes, z8.exps, width)
    slope = slope64(zv, act)
    exact = dy.double() * slope
    # dz is off by the slope's few last places of its largest term (1 + |z|), the result by half a step
    off = dy.double().abs() * 16 * 2.0 ** -23 * (1 + zv.abs())
    good = ~torch.isnan(zv)
    rows = good.all(1)   # a NaN times the unit matrix's zeros is a NaN in all of its row
    assert torch.equal(torch.isnan(got.dx), ~rows[:, None].expand_as(got.dx))
    assert ((got.dx.double() - exact).abs() <= off + 2.0 ** -8 * (exact.abs() + off))[rows].all()
    columns = good.all(0)
    # sums of `tokens` terms in fp32: at most tokens + 2 last places of the terms' magnitudes
    for have, terms in ((got.dbias, exact), (got.dscales, exact * zv)):
        mass = terms.abs().sum(0) + (off * (1 + zv.abs())).sum(0)
        assert ((have.double() - terms.sum(0)).abs() <= (off * (1 + zv.abs())).sum(0) + (tokens + 2) * 2.0 ** -23 * mass)[columns].all()
        assert torch.isnan(have[~columns]).all()
