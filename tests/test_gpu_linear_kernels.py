"""Activations, residuals and checkpoints in every kernel of the forward product, against 64-bit references.  Each case names the kernel that it is for, and
the library says which one the call takes."""
import ctypes

import pytest
import torch

import paper_2202_07471_b200 as sq
from linear_cases import ACTS, act64, decode64, encode64, gen, int_layer, pack, padded, real_layer, same_bits
from paper_2202_07471_b200 import linear

pytestmark = pytest.mark.gpu

FEW, FUSED, DENSE, WIDE = 1, 2, 3, 4


def _kernel(x, codes, cout, save):
    """What squant_linear_plan says of a call with these tensors."""
    ck = linear.CheckpointData(1 << 20, 1 << 20) if save else linear.CheckpointData(None, None)
    cin = x.shape[1]
    a = linear.LinearArgs(tokens=x.shape[0], cin=cin, cout=cout, dtype=int(x.dtype == torch.float16), act=0, flags=0 if codes.shape[1] == cin else sq.FLAG_PACK_INT4,
                          x=x.data_ptr(), x_stride=x.stride(0), codes=codes.data_ptr(), scales=1 << 20, y=1 << 20, y_stride=cout, z=ck)
    return linear._lib().squant_linear_plan(ctypes.byref(a))


# kernel, tokens, cin, cout, elements between rows, with a checkpoint
CASES = [(FEW, 5, 288, 200, 0, False), (FEW, 7, 288, 200, 1, False), (FEW, 70, 288, 200, 0, False), (FUSED, 3, 288, 200, 0, True), (FUSED, 20, 288, 200, 1, False),
         (FUSED, 100, 288, 77, 3, True), (FUSED, 140, 288, 200, 8, False), (FUSED, 256, 289, 201, 0, True), (DENSE, 300, 288, 200, 0, False),
         (DENSE, 513, 288, 77, 1, True), (DENSE, 600, 289, 201, 8, True), (WIDE, 2100, 72, 1700, 0, True), (WIDE, 2100, 71, 1701, 3, False)]


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("kernel,tokens,cin,cout,pad,save", CASES)
def test_activations(kernel, tokens, cin, cout, pad, save, dtype, bits, act):
    """|y - exact| <= half a step of the output (eps / 2 relative; fp16's smallest step is 2^-24) and what z's error makes of it: z is off by at most
    cin * 2^-23 of the sum of the products' magnitudes (each of cin additions, cut off or rounded, at most one last place of partial sums below
    that) and two roundings of the epilogue; slopes are at most 1.13, and the activation is a few last places off (16 * 2^-23 of |z|).  The checkpoint's
    value is half a step from z, the step that of the group's largest value, which z's error may move by a factor of two."""
    codes, scales = real_layer(cin, cout, bits, 5)
    stored = pack(codes) if bits == 4 else codes
    x, _ = padded(torch.randn((tokens, cin), generator=gen(6), device="cuda").to(dtype), pad)
    bias = torch.randn((cout,), generator=gen(7), device="cuda")
    s = scales.double()
    z = (x.double() @ codes.double().T) * s + bias.double()
    z_off = (cin + 2) * 2.0 ** -23 * ((x.double().abs() @ codes.double().abs().T) * s + bias.double().abs())
    assert _kernel(x, stored, cout, save) == kernel
    for with_residual in (False, True):
        res = padded(torch.randn((tokens, cout), generator=gen(8), device="cuda").to(dtype), pad)[0] if with_residual else None
        got = sq.squant_linear(x, stored, scales, bias, residual=res, act=act, pack_int4=bits == 4, checkpoint=save)
        y, z8 = got if save else (got, None)
        r = 0.0 if res is None else res.double()
        exact = act64(z, act) + r
        off = 1.13 * z_off + 16 * 2.0 ** -23 * (z.abs() + abs(r))
        bound = off + torch.finfo(dtype).eps / 2 * (exact.abs() + off) + (2.0 ** -25 if dtype == torch.float16 else 0)
        worst = ((y.double() - exact).abs() / bound).max().item()
        assert worst <= 1
        if save:
            group = torch.nn.functional.pad((z.abs() + z_off), (0, -cout % 32)).reshape(tokens, -1, 32).amax(2)
            step = torch.exp2(torch.floor(torch.log2(group)) - 6).repeat_interleave(32, 1)[:, :cout]
            # codes end at 127, so a value of the format between 127.5 and 128 steps, which a group's largest may be, is up to a step off: 128 - 127
            far = torch.where(z.abs() + z_off > 127.5 * step, step, step / 2)
            wrong = (decode64(z8.codes, z8.exps, cout) - z).abs() > far + z_off
            assert not wrong.any().item()
            assert cout % 32 == 0 or (z8.codes[:, cout:] == 0).all()


@pytest.mark.parametrize("act,lowest", [("gelu", -12.9), ("silu", -87.0)])
@pytest.mark.parametrize("kernel,tokens,save", [(FEW, 3, False), (FUSED, 40, True), (DENSE, 300, False)])
def test_tails_of_activations(kernel, tokens, save, act, lowest):
    """A channel's only product is one times one code of 1 or -1, so that z is the scale or its negative to the bit.  Far down the activation keeps its relative
    accuracy: half a step of bf16, and 3e-5 for expf of arguments down to -87 (2 + 1.16 * 87 last places, taken twice)."""
    cout = 1024
    want_z = torch.linspace(lowest, -lowest, cout, device="cuda")
    codes = torch.zeros((cout, 32), dtype=torch.int8, device="cuda")
    codes[:, 5] = torch.sign(want_z).to(torch.int8)
    x = torch.zeros((tokens, 32), dtype=torch.bfloat16, device="cuda")
    x[:, 5] = 1
    assert _kernel(x, codes, cout, save) == kernel
    y = sq.squant_linear(x, codes, want_z.abs(), act=act, checkpoint=save)
    exact = act64(want_z.double(), act).expand(tokens, cout)
    worst = (((y[0] if save else y).double() - exact).abs() / exact.abs()).max().item()
    assert worst <= 2.0 ** -8 + 3e-5


# up to eight tokens whose rows start anywhere, either side of the line for them
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("kernel,tokens,cin,cout,pad", [(FEW, 8, 2048, 4096, 1), (FUSED, 2, 2056, 4096, 1), (FUSED, 8, 2049, 4100, 0), (FUSED, 3, 16384, 40, 3), (FEW, 5, 2047, 70, 0)])
def test_few_tokens_of_rows_that_start_anywhere(kernel, tokens, cin, cout, pad, bits):
    codes, scales = int_layer(cin, cout, bits, 1)
    stored = pack(codes) if bits == 4 else codes
    x, _ = padded(torch.randint(-3, 4, (tokens, cin), generator=gen(2), device="cuda").bfloat16(), pad)
    assert _kernel(x, stored, cout, False) == kernel
    want = ((x.double() @ codes.double().T) * scales.double()).to(torch.bfloat16)
    n = sq.squant_launch_count()
    assert same_bits(sq.squant_linear(x, stored, scales, pack_int4=bits == 4) + 0.0, want + 0.0)
    assert sq.squant_launch_count() == n + (1 if kernel == FEW else 2)
    one = x[1:2]   # a row that starts off 16 bytes, alone
    assert same_bits(sq.squant_linear(one, stored, scales, pack_int4=bits == 4) + 0.0, want[1:2] + 0.0)


@pytest.mark.parametrize("kernel,tokens,cin,cout", [(FUSED, 9, 64, 33), (FUSED, 256, 128, 257), (DENSE, 257, 100, 33), (DENSE, 300, 128, 200), (DENSE, 513, 64, 1001),
                                                    (WIDE, 2100, 72, 1700), (WIDE, 2100, 72, 1663)])
def test_checkpoints_of_integers_are_exact(kernel, tokens, cin, cout):
    codes, scales = int_layer(cin, cout, 8, 11)
    x = torch.randint(-3, 4, (tokens, cin), generator=gen(12), device="cuda").bfloat16()
    bias = torch.randint(-9, 10, (cout,), generator=gen(13), device="cuda").float()
    assert _kernel(x, codes, cout, True) == kernel
    y, z = sq.squant_linear(x, codes, scales, bias, act="relu", checkpoint=True)
    exact = (x.double() @ codes.double().T) * scales.double() + bias.double()
    q, e = encode64(exact)
    assert torch.equal(z.exps, e) and torch.equal(z.codes, q)
    assert same_bits(y + 0.0, exact.clamp(min=0).to(torch.bfloat16) + 0.0)
    # a row with an infinity and one with a NaN
    x[1, 3], x[5, 0] = float("inf"), float("nan")
    _, z = sq.squant_linear(x, codes, scales, bias, checkpoint=True)
    rest = [i for i in range(tokens) if i not in (1, 5)]
    assert (z.exps[[1, 5]] == 255).all() and (z.codes[[1, 5]] == 0).all()
    assert torch.equal(z.exps[rest], e[rest]) and torch.equal(z.codes[rest], q[rest])


def test_many_calls_on_two_streams_without_a_wait():
    """Kernels that take all of a multiprocessor's tensor memory and kernels that share it, from two streams, queued far ahead."""
    codes, scales = real_layer(1024, 1024, 8, 1)
    x = torch.randn((300, 1024), generator=gen(2), device="cuda").bfloat16()
    x8 = sq.squant_checkpoint(x)

    def calls(tokens):
        y, z = sq.squant_linear(x[:tokens], codes, scales, act="gelu", checkpoint=True)
        part = sq.Checkpoint(x8.codes[:tokens], x8.exps[:tokens], 1024)
        g = sq.squant_linear_backward(y, codes, scales, act="gelu", z=z, x=part, dweight=True, dbias=True)
        return y, z.codes, g.dx, g.dweight, g.dbias

    wants = [[t.clone() for t in calls(tokens)] for tokens in (64, 300)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    last = [None, None]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for i in range(200):
        for k, s in enumerate(streams):
            with torch.cuda.stream(s):
                last[k] = calls((64, 300)[(i + k) % 2])
    torch.cuda.synchronize()
    for k in range(2):
        assert all(same_bits(a, b) for a, b in zip(last[k], wants[(199 + k) % 2]))
    sq.squant_device_status()
