"""The linear operators as a program uses them: with the quantizer, in a training step, on other streams, in graphs, at the edges."""
import math
import os
import subprocess
import sys
import threading

import pytest
import torch

import paper_2202_07471_b200 as sq
from linear_cases import act64, decode64, encode64, gen, int_layer, pack, padded, real_layer, same_bits, slope64
from paper_2202_07471_b200 import binding, linear

pytestmark = pytest.mark.gpu


def _x(tokens, cin, seed=1, dtype=torch.bfloat16):
    return torch.randint(-3, 4, (tokens, cin), generator=gen(seed), device="cuda").to(dtype)


def _want(x, codes, scales, bias=None):
    z = (x.double() @ codes.double().T) * scales.double()
    return z if bias is None else z + bias.double()


@pytest.mark.parametrize("tokens,save,launches", [(1, False, 1), (8, False, 1), (8, True, 1), (9, False, 1), (256, True, 1), (257, False, 2), (600, True, 2)])
def test_kernels_of_a_forward_call(tokens, save, launches):
    codes, scales = int_layer(128, 96, 8, 3)
    x = _x(tokens, 128)
    n = sq.squant_launch_count()
    sq.squant_linear(x, codes, scales, checkpoint=save)
    assert sq.squant_launch_count() == n + launches


# more steps of the contraction than a tile's stages, shared by several thread blocks; several tiles a thread block
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("tokens,cin,cout", [(5, 4096, 300), (16, 4096, 512), (40, 4096, 1100), (64, 11008, 256), (100, 4096, 512), (128, 2048, 1000), (200, 1500, 700), (700, 256, 9000),
                                             (40, 4096, 2200), (64, 11008, 1100), (100, 4096, 1500), (128, 4096, 1400), (24, 8192, 4096)])
def test_calls_repeat_to_the_bit(tokens, cin, cout, bits):
    codes, scales = int_layer(cin, cout, bits, 1)
    x = _x(tokens, cin)
    stored = pack(codes) if bits == 4 else codes
    want = _want(x, codes, scales).to(torch.bfloat16)
    bad = sum(not same_bits(sq.squant_linear(x, stored, scales, pack_int4=bits == 4), want) for _ in range(100))
    assert bad == 0
    sq.squant_device_status()


def test_many_calls_without_a_wait():
    """Launches of several kernels that fill the GPU, queued far ahead."""
    codes, scales = real_layer(1024, 1024, 8, 1)
    dy = torch.randn((1024, 1024), generator=gen(2), device="cuda").bfloat16()
    x8, z8 = sq.squant_checkpoint(dy), sq.squant_checkpoint(dy * 0.5)
    first = sq.squant_linear_backward(dy, codes, scales, act="gelu", z=z8, x=x8, dweight=True, dbias=True, dscales=True)
    for _ in range(600):
        last = sq.squant_linear_backward(dy, codes, scales, act="gelu", z=z8, x=x8, dweight=True, dbias=True, dscales=True)
    for a, b in ((first.dx, last.dx), (first.dweight, last.dweight), (first.dbias, last.dbias), (first.dscales, last.dscales)):
        assert same_bits(a, b)
    sq.squant_device_status()


@pytest.mark.parametrize("act", ["none", "silu"])
def test_no_tokens(act):
    codes, scales = real_layer(64, 40, 8, 1)
    x = torch.empty((0, 64), device="cuda", dtype=torch.bfloat16)
    y, z = sq.squant_linear(x, codes, scales, act=act, checkpoint=True)
    assert y.shape == (0, 40) and z.codes.shape == (0, 64) and z.exps.shape == (0, 2)
    x8 = sq.squant_checkpoint(x)
    assert sq.squant_checkpoint_restore(x8).shape == (0, 64)
    g = sq.squant_linear_backward(y, codes, scales, act=act, z=z, x=x8, dweight=True, dbias=True, dscales=True)
    assert g.dx.shape == (0, 64)
    for t in (g.dweight, g.dbias, g.dscales):
        assert (t == 0).all()
    assert sq.squant_linear(torch.empty((2, 0, 64), device="cuda", dtype=torch.bfloat16), codes, scales).shape == (2, 0, 40)


def test_leading_dimensions():
    codes, scales = int_layer(96, 40, 8, 1)
    x = _x(6 * 5, 96).view(2, 3, 5, 96)
    res = _x(6 * 5, 40, 2).view(2, 3, 5, 40)
    want = _want(x.view(30, 96), codes, scales).view(2, 3, 5, 40)
    assert same_bits(sq.squant_linear(x, codes, scales, residual=res), (want + res.double()).to(torch.bfloat16))
    one = sq.squant_linear(x[0, 0, 0], codes, scales)
    assert one.shape == (40,) and same_bits(one, want[0, 0, 0].to(torch.bfloat16))
    g = sq.squant_linear_backward(res, codes, scales, x=sq.squant_checkpoint(x), dweight=True)
    assert g.dx.shape == x.shape and g.dweight.shape == (40, 96)
    # codes of a 1x1 convolution's weights
    c4 = codes.view(40, 96, 1, 1)
    assert same_bits(sq.squant_linear(x, c4, scales), want.to(torch.bfloat16))
    assert same_bits(sq.squant_linear_backward(res, c4, scales).dx, g.dx)
    # a slice of heads: rows that lie apart
    wide = torch.zeros((30, 3, 96), device="cuda", dtype=torch.bfloat16)
    wide[:, 1] = x.view(30, 96)
    assert same_bits(sq.squant_linear(wide[:, 1], codes, scales), want.view(30, 40).to(torch.bfloat16))


@pytest.mark.parametrize("tokens", [5, 40, 300])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_residual_in_place_and_what_lies_behind(tokens, dtype):
    codes, scales = int_layer(64, 72, 4, 1)
    scales = scales * 2.0 ** -6
    x = _x(tokens, 64, dtype=dtype)
    buf = _x(tokens + 50, 72 + 9, 2, dtype)
    before = buf.clone()
    y = buf[:tokens, :72]
    want = (_want(x, codes, scales) + y.double()).to(dtype)
    got = sq.squant_linear(x, pack(codes), scales, residual=y, out=y, pack_int4=True)
    assert got.data_ptr() == y.data_ptr() and same_bits(y, want)
    assert torch.equal(buf[tokens:], before[tokens:]) and torch.equal(buf[:, 72:], before[:, 72:])


@pytest.mark.parametrize("tokens", [4, 40, 300])
def test_infinities_and_nan_stay_in_their_row(tokens):
    codes, scales = int_layer(100, 40, 8, 1)
    x = _x(tokens, 100)
    want = _want(x, codes, scales).to(torch.bfloat16)
    x[1, 3], x[2, 99] = float("nan"), float("inf")
    y, z = sq.squant_linear(x, codes, scales, checkpoint=True)
    rest = [i for i in range(tokens) if i not in (1, 2)]
    assert same_bits(y[rest], want[rest])
    assert torch.isnan(y[1]).all()
    finite = codes[:, 99] == 0                       # inf * 0
    assert torch.isnan(y[2][finite]).all() and torch.isinf(y[2][~finite]).all()
    assert (z.exps[1] == 255).all() and (z.exps[rest] != 255).all()


def test_poisoned_groups_of_checkpoints():
    codes, scales = real_layer(96, 70, 8, 1)
    tokens = 140
    dy = torch.ones((tokens, 70), device="cuda", dtype=torch.bfloat16)
    x = torch.ones((tokens, 96), device="cuda", dtype=torch.bfloat16)
    z = torch.ones((tokens, 70), device="cuda", dtype=torch.bfloat16)
    x[17, 40], z[5, 69] = float("nan"), float("inf")
    g = sq.squant_linear_backward(dy, codes, scales, act="gelu", z=sq.squant_checkpoint(z), x=sq.squant_checkpoint(x), dweight=True, dbias=True, dscales=True)
    column, row = torch.zeros(96, dtype=torch.bool), torch.zeros(70, dtype=torch.bool)
    column[32:64], row[64:] = True, True
    bad = (column[None] | row[:, None]).cuda()
    assert torch.equal(torch.isnan(g.dweight), bad)
    assert torch.equal(torch.isnan(g.dbias).cpu(), row) and torch.equal(torch.isnan(g.dscales).cpu(), row)
    assert torch.isnan(g.dx[5]).all() and not torch.isnan(g.dx[6:]).any()


def test_streams():
    codes, scales = int_layer(512, 300, 8, 1)
    bias = torch.ones(300, device="cuda")
    xs = [_x(t, 512, t) for t in (3, 50, 300)]
    wants = [_want(x, codes, scales, bias) for x in xs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = []
    for x in xs:
        out.append(sq.squant_linear(x, codes, scales, bias, stream=side))
        with torch.cuda.stream(side):
            out.append(sq.squant_linear(x, codes, scales, bias))
            c = sq.squant_checkpoint(x)
        out.append(sq.squant_checkpoint_restore(c, stream=side))
    side.synchronize()
    for x, w, (a, b, r) in zip(xs, wants, zip(*[iter(out)] * 3)):
        assert same_bits(a, w.to(torch.bfloat16)) and same_bits(b, a) and same_bits(r + 0.0, x + 0.0)


def test_python_and_native_calls_agree(monkeypatch):
    codes, scales = real_layer(160, 96, 4, 1)
    stored = pack(codes)
    bias = torch.randn(96, generator=gen(2), device="cuda")
    x = torch.randn((300, 160), generator=gen(3), device="cuda").bfloat16()
    dy = torch.randn((300, 96), generator=gen(4), device="cuda").bfloat16()

    def run():
        y, z = sq.squant_linear(x, stored, scales, bias, residual=dy, act="silu", pack_int4=True, checkpoint=True)
        x8 = sq.squant_checkpoint(x)
        g = sq.squant_linear_backward(dy, stored, scales, bias, cin=160, act="silu", pack_int4=True, z=z, x=x8, dweight=True, dbias=True, dscales=True)
        return [y, z.codes, z.exps, x8.codes, x8.exps, sq.squant_checkpoint_restore(x8), g.dx, g.dweight, g.dbias, g.dscales]

    assert binding._marshal is not None and linear._native() is not None
    native = run()
    monkeypatch.setattr(binding, "_marshal", None)
    for a, b in zip(native, run()):
        assert same_bits(a, b)


def test_refusals():
    codes, scales = real_layer(64, 32, 8, 1)
    x = torch.zeros((4, 64), device="cuda", dtype=torch.bfloat16)
    dy = torch.zeros((4, 32), device="cuda", dtype=torch.bfloat16)
    n = sq.squant_launch_count()
    z8, x8 = encode64(dy), encode64(x)
    z8, x8 = sq.Checkpoint(*z8, 32), sq.Checkpoint(*x8, 64)
    for call in (lambda: sq.squant_linear(x.float(), codes, scales), lambda: sq.squant_linear(x, codes.float(), scales),
                 lambda: sq.squant_linear(x, codes[:, :63], scales), lambda: sq.squant_linear(x, codes, scales, pack_int4=True),
                 lambda: sq.squant_linear(x, codes, scales[:31]), lambda: sq.squant_linear(x, codes, scales.double()),
                 lambda: sq.squant_linear(x, codes, scales, torch.zeros(33, device="cuda")), lambda: sq.squant_linear(x, codes, scales.cpu()),
                 lambda: sq.squant_linear(x, codes, scales, act="tanh"), lambda: sq.squant_linear(x, codes, scales, residual=dy.half()),
                 lambda: sq.squant_linear(x, codes, scales, out=dy[:3]), lambda: sq.squant_linear(x.t(), codes, scales),
                 lambda: sq.squant_linear(x[:, ::2], codes[:, :32].contiguous(), scales), lambda: sq.squant_linear(x[:, :0], codes, scales),
                 lambda: sq.squant_checkpoint(x.half()), lambda: sq.squant_checkpoint_restore(sq.Checkpoint(x8.codes, x8.exps, 65)),
                 lambda: sq.squant_linear_backward(dy.half(), codes, scales), lambda: sq.squant_linear_backward(dy, codes, scales, act="relu"),
                 lambda: sq.squant_linear_backward(dy, codes, scales, dscales=True), lambda: sq.squant_linear_backward(dy, codes, scales, dweight=True),
                 lambda: sq.squant_linear_backward(dy, codes[:31], scales), lambda: sq.squant_linear_backward(dy, codes, scales, act="relu", z=x8),
                 lambda: sq.squant_linear_backward(dy, codes, scales, dweight=True, x=z8),
                 lambda: sq.squant_linear_backward(dy, pack(codes), scales, pack_int4=True),
                 lambda: sq.squant_linear_backward(dy, pack(codes), scales, cin=62, pack_int4=True),
                 lambda: sq.squant_linear(x, codes, scales, stream=torch.cuda.Stream(), act="x"),
                 lambda: sq.squant_linear(x, codes.view(-1), scales), lambda: sq.squant_linear_backward(dy, codes.view(-1), scales),
                 lambda: sq.squant_linear_backward(dy[0, 0], codes, scales, act="relu", z=z8)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: sq.squant_linear(x[:1].expand(4, 64), codes, scales),   # one row for all tokens
                 lambda: sq.squant_linear(x, codes[:0], scales[:0]), lambda: sq.squant_linear_backward(dy[:, :0].contiguous(), codes[:0], scales[:0]),
                 lambda: sq.squant_checkpoint_restore(sq.Checkpoint(x8.codes[1:], x8.exps[1:], 64))):   # exponents start on 2 bytes
        with pytest.raises((ValueError, sq.SquantError)):
            call()
    assert sq.squant_launch_count() == n


def _layer_pass(x, dy, stored, scales, bias, packed):
    y, z = sq.squant_linear(x, stored, scales, bias, act="gelu", pack_int4=packed, checkpoint=True)
    x8 = sq.squant_checkpoint(x)
    g = sq.squant_linear_backward(dy, stored, scales, bias, cin=x.shape[1], act="gelu", pack_int4=packed, z=z, x=x8, dweight=True, dbias=True, dscales=True)
    return y, g.dx, g.dweight, g.dbias, g.dscales


@pytest.mark.parametrize("tokens", [6, 90, 400])
def test_two_graphs_of_the_same_layer(tokens):
    """Each replay uses its own inputs and workspaces, in any order."""
    codes, scales = real_layer(200, 136, 4, 1)
    stored, bias = pack(codes), torch.randn(136, generator=gen(2), device="cuda")
    inputs = [(torch.randn((tokens, 200), generator=gen(s), device="cuda").bfloat16(), torch.randn((tokens, 136), generator=gen(s + 1), device="cuda").bfloat16())
              for s in (10, 20, 30)]
    want = [[t.clone() for t in _layer_pass(x, dy, stored, scales, bias, True)] for x, dy in inputs]
    static = [[t.clone() for t in inputs[0]] for _ in range(2)]
    graphs, outs = [], []
    for x, dy in static:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(_layer_pass(x, dy, stored, scales, bias, True))
        graphs.append(g)
    side = torch.cuda.Stream()
    for order in ((0, 1, 2), (2, 1, 0)):
        for which in order:
            for k in range(2):
                for a, b in zip(static[k], inputs[(which + k) % 3]):
                    a.copy_(b)
            side.wait_stream(torch.cuda.current_stream())
            graphs[0].replay()
            with torch.cuda.stream(side):
                graphs[1].replay()
            torch.cuda.current_stream().wait_stream(side)
            torch.cuda.synchronize()
            for k in range(2):
                for a, b in zip(outs[k], want[(which + k) % 3]):
                    assert same_bits(a, b)
    sq.squant_device_status()


@pytest.mark.parametrize("pack_int4", [False, True])
def test_with_the_quantizer(pack_int4):
    """Codes, scales and dequantized weights as the quantizer writes them: the layer is the product with the dequantized weights."""
    cin, cout, tokens = 320, 144, 70
    w = torch.randn((cout, cin), generator=gen(1), device="cuda") / math.sqrt(cin)
    b = sq.alloc_outputs(w, kernel_err=False, channel_err=False, pack_int4=pack_int4, dequant=True)
    flags = sq.FLAG_NARROW_RANGE | (sq.FLAG_PACK_INT4 if pack_int4 else 0)
    sq.squant_quantize_model([b], bits=4, flags=flags)
    x = torch.randn((tokens, cin), generator=gen(2), device="cuda").bfloat16()
    y = sq.squant_linear(x, b.codes, b.scales, pack_int4=pack_int4)
    exact = x.double() @ b.dequant.double().T
    mass = x.double().abs() @ b.dequant.double().abs().T
    # the dequantized weights are rounded (2^-24), the sum is off by up to cin + 1 last places of the terms' magnitudes, the output by half a step
    bound = (cin + 2) * 2.0 ** -23 * mass
    assert ((y.double() - exact).abs() <= bound + 2.0 ** -8 * (exact.abs() + bound)).all()


def test_training_steps():
    """Two layers, quantized anew before each step, trained through the 8-bit checkpoints: every gradient is that of the 64-bit
    formulas on the values the step holds, and the steps run in a row."""
    tokens, width, hidden = 96, 128, 200
    w = [torch.randn((hidden, width), generator=gen(1), device="cuda") / math.sqrt(width), torch.randn((width, hidden), generator=gen(2), device="cuda") / math.sqrt(hidden)]
    bias = [torch.zeros(hidden, device="cuda"), torch.zeros(width, device="cuda")]
    target = torch.randn((tokens, width), generator=gen(3), device="cuda")
    x = torch.randn((tokens, width), generator=gen(4), device="cuda").bfloat16()
    acts = ("gelu", "none")
    for _ in range(3):
        q = [sq.squant_quantize_layer(v, bits=8) for v in w]
        h, z1 = sq.squant_linear(x, q[0].codes, q[0].scales, bias[0], act=acts[0], checkpoint=True)
        y = sq.squant_linear(h, q[1].codes, q[1].scales, bias[1], residual=x)
        kept = [sq.squant_checkpoint(x), sq.squant_checkpoint(h)]
        dy = ((y.float() - target) / tokens).bfloat16()
        g2 = sq.squant_linear_backward(dy, q[1].codes, q[1].scales, bias[1], x=kept[1], dweight=True, dbias=True)
        g1 = sq.squant_linear_backward(g2.dx, q[0].codes, q[0].scales, bias[0], act=acts[0], z=z1, x=kept[0], dweight=True, dbias=True)
        for g, up, ck, z, act, layer in ((g2, dy, kept[1], None, "none", q[1]), (g1, g2.dx, kept[0], z1, "gelu", q[0])):
            dz = up.double()
            slack = dz.abs() * 2.0 ** -8
            if z is not None:
                zv = decode64(z.codes, z.exps, z.features)
                slope = slope64(zv, act)
                slack = dz.abs() * (slope.abs() * 2.0 ** -8 + 16 * 2.0 ** -23 * (1 + zv.abs()))
                dz = dz * slope
            xv = decode64(ck.codes, ck.exps, ck.features)
            exact = dz.T @ xv
            off = slack.T @ xv.abs() + (tokens + 2) * 2.0 ** -23 * (dz.abs().T @ xv.abs())
            assert ((g.dweight.double() - exact).abs() <= off + 2.0 ** -8 * (exact.abs() + off)).all()
            c = layer.codes.double() * layer.scales.double()[:, None]
            exact = dz @ c
            off = slack @ c.abs() + (c.shape[0] + 2) * 2.0 ** -23 * (dz.abs() @ c.abs())
            assert ((g.dx.double() - exact).abs() <= off + 2.0 ** -8 * (exact.abs() + off)).all()
        for v, b, g in ((w[0], bias[0], g1), (w[1], bias[1], g2)):
            v -= 0.05 * g.dweight.float()
            b -= 0.05 * g.dbias
    sq.squant_device_status()


@pytest.mark.parametrize("act", ["gelu", "silu"])
def test_gradients_against_differences(act):
    """Along a direction of x, bias and scales the 64-bit forward formula changes as the gradients say.  zhat and xhat are exact here (integers of
    at most seven bits times a power of two), so the gradients' own error is that of dz in bf16 (2^-8 of each term) and of fp32 sums; the
    central difference is off by h^2 / 6 times the third derivative along the direction (h = 2^-10: below 1e-5 of the terms)."""
    tokens, cin, cout = 60, 64, 48
    codes, scales = int_layer(cin, cout, 4, 1)
    scales = torch.full_like(scales, 2.0 ** -6)
    x = torch.randint(-2, 3, (tokens, cin), generator=gen(2), device="cuda").double()
    x[:, 8:] = 0                                                            # |z| <= 2 * 8 * 8 / 64 = 2, in units of 1 / 64: 128 steps, 127 asserted
    bias = torch.zeros(cout, device="cuda", dtype=torch.float64)
    dy = torch.randint(-3, 4, (tokens, cout), generator=gen(3), device="cuda").double()
    dirs = [torch.randn(t.shape, generator=gen(s), device="cuda", dtype=torch.float64) for s, t in ((4, x), (5, bias), (6, scales))]
    c, s0 = codes.double(), scales.double()
    z = (x @ c.T) * s0 + bias
    q, e = encode64(z)
    assert torch.equal(decode64(q, e, cout), z)
    loss = lambda h: (dy * act64(((x + h * dirs[0]) @ c.T) * (s0 + h * 2.0 ** -6 * dirs[2]) + bias + h * dirs[1], act)).sum()
    h = 2.0 ** -10
    slope_along = (loss(h) - loss(-h)) / (2 * h)
    g = sq.squant_linear_backward(dy.bfloat16(), codes, scales, bias.float(), act=act, z=sq.Checkpoint(q, e, cout), dbias=True, dscales=True)
    got = (g.dx.double() * dirs[0]).sum() + (g.dbias.double() * dirs[1]).sum() + (g.dscales.double() * 2.0 ** -6 * dirs[2]).sum()
    dz = (dy * slope64(z, act)).abs()
    dx_mass = (dz * s0) @ c.abs()
    bound = (2.0 ** -8 * dx_mass + 2.0 ** -8 * dx_mass) * dirs[0].abs()
    # |third derivative| of gelu and silu is below 2, of z along the direction u: u^3 dy / 6 * h^2, and second-order terms of x times scales alike
    u = (dirs[0] @ c.T).abs() * s0 + (x @ c.T).abs() * 2.0 ** -6 * dirs[2].abs() + dirs[1].abs() + (dirs[0] @ c.T).abs() * 2.0 ** -6 * dirs[2].abs()
    rest = (dy.abs() * (1 + u) ** 3).sum() * h * h + 2.0 ** -16 * (dz * (dirs[1].abs() + (z.abs() + 1) * dirs[2].abs())).sum()
    assert (got - slope_along).abs() <= bound.sum() + rest


@pytest.mark.parametrize("tokens", [2100, 6])
def test_offsets_beyond_32_bits(tokens):
    """Rows half a billion elements apart at most: x, y, residual, dy beyond 2^31 elements."""
    stride = (1 << 31) // (tokens - 1) // 8 * 8 + 64
    codes, scales = int_layer(72, 40, 8, 1)
    xb = torch.empty(tokens * stride, dtype=torch.bfloat16, device="cuda")
    yb = torch.empty(tokens * stride, dtype=torch.bfloat16, device="cuda")
    x = xb.as_strided((tokens, 72), (stride, 1))
    y = yb.as_strided((tokens, 40), (stride, 1))
    x.copy_(_x(tokens, 72))
    y.copy_(_x(tokens, 40, 2))
    want = (_want(x, codes, scales) + y.double()).to(torch.bfloat16)
    sq.squant_linear(x, codes, scales, residual=y, out=y)
    assert same_bits(y, want)
    y.copy_(_x(tokens, 40, 2))
    g = sq.squant_linear_backward(y, codes, scales, x=sq.squant_checkpoint(x), dweight=True, dbias=True)
    x8 = encode64(x)
    assert same_bits(g.dweight + 0.0, (y.double().T @ decode64(*x8, 72)).to(torch.bfloat16) + 0.0)
    assert torch.equal(g.dbias.double(), y.double().sum(0))
    sq.squant_device_status()


@pytest.mark.parametrize("tokens", [3, 20])
def test_codes_beyond_32_bits(tokens):
    cin, cout = 32768, 65600   # 2.15e9 codes
    codes = torch.randint(-128, 128, (64, cin), generator=gen(1), device="cuda", dtype=torch.int32).to(torch.int8).repeat(cout // 64, 1)
    codes[-1] = 3
    scales = torch.full((cout,), 2.0 ** -8, device="cuda")
    x = _x(tokens, cin)
    y = sq.squant_linear(x, codes, scales)
    want = (x.double() @ codes[-64:].double().T) * 2.0 ** -8
    mass = (x.double().abs() @ codes[-64:].double().abs().T).max()
    assert mass < 2 ** 24   # sums are exact in any order
    assert same_bits(y[:, -64:], want.to(torch.bfloat16)) and same_bits(y[:, :63], want[:, :63].to(torch.bfloat16))


def test_calls_from_other_threads():
    """A thread's first work on the GPU is a call (each kind of it), and four threads call at once on streams of their own."""
    codes, scales = real_layer(256, 136, 4, 1)
    stored, bias = pack(codes), torch.randn(136, generator=gen(2), device="cuda")
    cases = []
    for tokens in (6, 64, 400):
        x, dy = torch.randn((tokens, 256), generator=gen(tokens), device="cuda").bfloat16(), torch.randn((tokens, 136), generator=gen(9), device="cuda").bfloat16()
        cases.append((x, dy, [t.clone() for t in _layer_pass(x, dy, stored, scales, bias, True)]))
    torch.cuda.synchronize()
    failed = []

    def guarded(work):
        def run():
            try:
                work()
            except Exception as e:
                failed.append(e)
        return run

    def first_call(x, dy, want):
        out = torch.empty_like(want[0])

        def work():
            assert same_bits(sq.squant_linear(x, stored, scales, bias, act="gelu", pack_int4=True, out=out), want[0])
        return work

    def many(k):
        def work():
            side = torch.cuda.Stream()
            with torch.cuda.stream(side):
                for i in range(60):
                    x, dy, want = cases[(i + k) % 3]
                    got = _layer_pass(x, dy, stored, scales, bias, True)
                    assert all(same_bits(a, b) for a, b in zip(got, want))
        return work

    for case in cases:
        t = threading.Thread(target=guarded(first_call(*case)))
        t.start()
        t.join()
    threads = [threading.Thread(target=guarded(many(k))) for k in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed, failed
    sq.squant_device_status()


@pytest.mark.parametrize("tokens", [6, 90, 400])
def test_first_calls_of_a_process_in_a_capture(tokens):
    """Kernels are loaded and set up while a graph is being recorded."""
    here = os.path.dirname(os.path.abspath(__file__))
    program = f"""
import sys
sys.path[:0] = [{here!r}, {os.path.dirname(here)!r}]
import torch
import paper_2202_07471_b200 as sq
from linear_cases import gen, pack, real_layer, same_bits
codes, scales = real_layer(200, 136, 4, 1)
stored, bias = pack(codes), torch.randn(136, generator=gen(2), device="cuda")
x, dy = torch.randn(({tokens}, 200), generator=gen(3), device="cuda").bfloat16(), torch.randn(({tokens}, 136), generator=gen(4), device="cuda").bfloat16()
def work():
    y, z = sq.squant_linear(x, stored, scales, bias, act="gelu", pack_int4=True, checkpoint=True)
    x8 = sq.squant_checkpoint(x)
    g = sq.squant_linear_backward(dy, stored, scales, bias, cin=200, act="gelu", pack_int4=True, z=z, x=x8, dweight=True, dbias=True, dscales=True)
    return y, sq.squant_linear(x[:3], stored, scales, pack_int4=True), sq.squant_checkpoint_restore(x8), g.dx, g.dweight, g.dbias, g.dscales
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    out = work()
graph.replay()
assert all(same_bits(a, b) for a, b in zip(out, work()))
sq.squant_device_status()
"""
    done = subprocess.run([sys.executable, "-c", program], capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, done.stderr[-2000:]


def test_more_rows_than_a_launch_takes():
    """2^30 rows: a launch indexes fewer than 2^31 pieces of rows."""
    rows = 1 << 30
    if torch.cuda.mem_get_info()[0] < 80 << 30:
        pytest.skip("needs 80 GB")
    base = torch.randint(-127, 128, (1000003, 1), generator=gen(1), device="cuda").to(torch.bfloat16)
    x = base.repeat(rows // 1000003 + 1, 1)[:rows]
    c = sq.squant_checkpoint(x)
    assert torch.equal(sq.squant_checkpoint_restore(c), x)
    assert (c.codes[::99991, 1:] == 0).all()
    del c, x
    base = torch.randint(-3, 4, (1000003, 9), generator=gen(2), device="cuda").to(torch.bfloat16)
    x = base.repeat(rows // 1000003 + 1, 1)[:rows]   # rows of 18 bytes, which are copied first
    codes, scales = int_layer(9, 1, 8, 3)
    want = _want(base, codes, scales).to(torch.bfloat16).repeat(rows // 1000003 + 1, 1)[:rows]
    assert torch.equal(sq.squant_linear(x, codes, scales), want)
    sq.squant_device_status()
