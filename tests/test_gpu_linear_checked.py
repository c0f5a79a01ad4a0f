"""The linear operators' checked build and their failure path."""
import pytest
import torch

import paper_2202_07471_b200 as sq
from linear_cases import ACTS, gen, int_layer, pack, padded, real_layer, same_bits
from paper_2202_07471_b200 import build as lib_build

pytestmark = pytest.mark.gpu


def _status():
    """Error code of the device's status, 0 for none."""
    try:
        sq.squant_device_status()
        return 0
    except sq.SquantError as e:
        return e.code


@pytest.fixture
def checked_build():
    sq.use_library(lib_build.LIB_DEBUG)
    try:
        yield
    finally:
        sq.squant_debug_linear_wait_limit(-1)
        sq.use_library(None)


def test_a_wait_that_runs_out_is_reported_once():
    assert _status() == 0
    sq.squant_debug_linear_wait_expires(64)
    assert _status() == -10 and _status() == 0
    with pytest.raises(sq.SquantError):
        sq.squant_debug_linear_wait_expires(0)
    # next to the quantizer's
    sq.squant_debug_linear_wait_expires(1)
    sq.squant_debug_set_status(1)
    assert _status() == -10 and _status() == 0
    assert not sq.squant_debug_linear_wait_limit(0)   # the regular build's limit stays
    codes, scales = int_layer(256, 96, 8, 1)
    x = torch.randint(-3, 4, (300, 256), generator=gen(2), device="cuda").bfloat16()
    y = sq.squant_linear(x, codes, scales)
    assert _status() == 0 and same_bits(y, ((x.double() @ codes.double().T) * scales.double()).to(torch.bfloat16))


# clusters of eight, one thread block a tile, two row tiles; pairs with fewer and more steps than stages, several tiles a pair
@pytest.mark.parametrize("tokens,cin,cout", [(40, 4096, 300), (200, 64, 1000), (256, 1500, 700), (300, 64, 96), (300, 4096, 300), (1500, 1024, 9000)])
@pytest.mark.parametrize("bits", [4, 8])
def test_calls_that_give_up_end_and_leave_the_gpu_usable(checked_build, tokens, cin, cout, bits):
    """Without a try, every kernel that waits for copies, conversions or products gives up: the call returns, the status says so, and the same calls
    with the regular limit are right.  With one try (4 us) some waits give up in the middle of a tile, or none does."""
    codes, scales = int_layer(cin, cout, bits, 1)
    stored = pack(codes) if bits == 4 else codes
    x = torch.randint(-3, 4, (tokens, cin), generator=gen(2), device="cuda").bfloat16()
    dy = torch.randint(-1, 2, (tokens, cout), generator=gen(3), device="cuda").bfloat16()
    x8 = sq.squant_checkpoint(x)
    ones = torch.ones_like(scales)

    def call():
        y, _ = sq.squant_linear(x, stored, ones, pack_int4=bits == 4, checkpoint=True)
        g = sq.squant_linear_backward(dy, stored, ones, cin=cin, pack_int4=bits == 4, x=x8, dweight=True)
        return y, g.dx, g.dweight

    c = codes.double()
    wants = [t.to(torch.bfloat16) for t in (x.double() @ c.T, dy.double() @ c, dy.double().T @ x.double())]
    for tries in (0, 1, 0):
        assert sq.squant_debug_linear_wait_limit(tries)
        call()
        assert _status() in ((-10,) if tries == 0 else (-10, 0))
        assert sq.squant_debug_linear_wait_limit(-1)
        got = call()
        assert _status() == 0
        for a, b in zip(got, wants):
            assert same_bits(a + 0.0, b + 0.0)


# every kernel and tile: few tokens with rows on 32, 16 and fewer bytes; thread blocks of one tile; one and two row tiles; wide tiles; long contractions
SHAPES = [(1, 1, 1, 0), (8, 256, 64, 0), (7, 136, 50, 8), (5, 33, 70, 1), (16, 1000, 257, 24), (30, 96, 31, 32), (64, 512, 100, 0), (256, 64, 100, 0), (9, 61, 33, 3), (100, 3000, 64, 0),
          (129, 256, 255, 1), (200, 31, 1001, 0), (256, 4096, 300, 0), (257, 320, 384, 0), (300, 1537, 1001, 3), (700, 72, 33, 0), (2100, 72, 1700, 0), (40, 70000, 70, 0),
          (300, 70000, 40, 5), (70000, 40, 72, 0), (3, 530000, 9, 0)]


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("tokens,cin,cout,pad", SHAPES)
def test_indices_stay_in_bounds(tokens, cin, cout, pad, bits):
    """No check of the checked build fails, and its results are the regular build's."""
    codes, scales = real_layer(cin, cout, bits, 5)
    stored = pack(codes) if bits == 4 else codes
    x = padded(torch.randn((tokens, cin), generator=gen(6), device="cuda").bfloat16(), pad)[0]
    dy = padded(torch.randn((tokens, cout), generator=gen(7), device="cuda").bfloat16(), pad)[0]
    bias = torch.randn(cout, generator=gen(8), device="cuda")

    def calls():
        out = []
        for act in ACTS:
            for save in (False, True):
                got = sq.squant_linear(x, stored, scales, bias, residual=dy, act=act, pack_int4=bits == 4, checkpoint=save)
                out += [got[0], got[1].codes, got[1].exps] if save else [got]
            x8, z8 = sq.squant_checkpoint(x), got[1]
            g = sq.squant_linear_backward(dy, stored, scales, bias, cin=cin, act=act, pack_int4=bits == 4, z=z8, x=x8, dweight=True, dbias=True, dscales=True)
            out += [x8.codes, x8.exps, sq.squant_checkpoint_restore(x8), g.dx, g.dweight, g.dbias, g.dscales]
        half = sq.squant_linear(x.half(), stored, scales, bias, pack_int4=bits == 4)
        return out + [half, sq.squant_linear_backward(dy, stored, scales, cin=cin, pack_int4=bits == 4, dbias=True).dbias]

    want = calls()
    assert sq.squant_debug_violations()[:2] == (False, 0)
    sq.use_library(lib_build.LIB_DEBUG)
    try:
        sq.squant_debug_violations()
        got = calls()
        checked, failed, site = sq.squant_debug_violations()
        assert checked and failed == 0, (failed, site)
    finally:
        sq.use_library(None)
    assert all(same_bits(a, b) for a, b in zip(got, want))
    assert _status() == 0
