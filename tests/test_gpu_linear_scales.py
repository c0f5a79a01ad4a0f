"""The gradient of the scales against the layer's own, where channels are of different sizes: what the documentation says of it."""
import math

import pytest
import torch

import paper_2202_07471_b200 as sq
from linear_cases import gen, pack

pytestmark = pytest.mark.gpu


def _step(v):
    """Step of the checkpoint's group of 32 that a value lies in."""
    top = torch.frexp(v.abs().reshape(v.shape[0], -1, 32).amax(2)).exponent - 1
    return torch.exp2((top - 6).double()).repeat_interleave(32, 1)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("spread", [0.0, 0.3, 1.0, 2.0])
@pytest.mark.parametrize("shift", [0.0, 1.0])
def test_of_channels_of_different_sizes(spread, shift, bits):
    tokens, cin, cout = 512, 256, 256
    g = gen(1)
    w = torch.randn((cout, cin), generator=g, device="cuda") / math.sqrt(cin) * torch.exp(spread * torch.randn((cout, 1), generator=g, device="cuda"))
    q = sq.squant_quantize_layer(w, bits=bits)
    codes, scales = q.codes.double(), q.scales.double()
    stored = pack(q.codes) if bits == 4 else q.codes
    bias = shift * torch.randn(cout, generator=g, device="cuda")
    x = torch.randn((tokens, cin), generator=g, device="cuda").bfloat16()
    dy = torch.randn((tokens, cout), generator=g, device="cuda").bfloat16()
    _, z8 = sq.squant_linear(x, stored, q.scales, bias, pack_int4=bits == 4, checkpoint=True)
    got = sq.squant_linear_backward(dy, stored, q.scales, bias, cin=cin, pack_int4=bits == 4, z=z8, x=sq.squant_checkpoint(x), dweight=True, dscales=True)
    u = x.double() @ codes.T
    z = u * scales + bias.double()
    dz = dy.double()
    exact = (dz * u).sum(0)
    # z is cin + 2 last places of its terms off before it is rounded to half a step (a step beyond 127.5 of them); a moved z may move the step's
    # power of two only where the group's largest is next to one, and half of the doubled step is counted there; then all is divided by the scale
    z_off = (cin + 2) * 2.0 ** -23 * ((x.double().abs() @ codes.abs().T) * scales + bias.double().abs())
    step = _step(z)
    wide = z.abs().reshape(tokens, -1, 32).amax(2).repeat_interleave(32, 1) + z_off >= 128 * step
    off = torch.where(wide | (z.abs() + z_off > 127.5 * step), step, step / 2) + z_off
    place = (tokens + 4) * 2.0 ** -23   # of the fp32 sum and of zhat - bias
    bound = (dz.abs() * (off + place * (z.abs() + off + bias.double().abs()))).sum(0) / scales
    assert ((got.dscales.double() - exact).abs() <= bound).all()
    # from the input: its checkpoint is half a step off (bf16 values are never beyond 127.5 steps), dweight is rounded by half a place
    from_input = (got.dweight.double() * codes).sum(1)
    xv = x.double()
    each = dz.abs().T @ (_step(xv) / 2 + (tokens + 2) * 2.0 ** -23 * xv.abs())
    each = each + 2.0 ** -8 * ((dz.T @ xv).abs() + each)
    assert ((from_input - exact).abs() <= (each * codes.abs()).sum(1)).all()

    def relative(a):
        return ((a - exact).norm() / exact.norm()).item()

    print(f"bits {bits} spread {spread} shift {shift}: {relative(got.dscales.double()):.4f} from z, {relative(from_input):.4f} from the input")
    # as documented; a rounding to a grid of steps leaves 0.29 of a step on average, the bounds above are the worst case's
    if spread <= 0.3:
        assert relative(got.dscales.double()) < 0.03
    assert relative(from_input) < 0.02
