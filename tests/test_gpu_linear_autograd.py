"""The linear operators next to autograd: what they refuse, and a torch.autograd.Function around them."""
import pytest
import torch

import paper_2202_07471_b200 as sq
from linear_cases import gen, pack, real_layer, same_bits
from paper_2202_07471_b200 import binding, linear

pytestmark = pytest.mark.gpu


@pytest.fixture(params=["native", "python"])
def path(request, monkeypatch):
    if request.param == "python":
        monkeypatch.setattr(binding, "_marshal", None)
    else:
        assert binding._marshal is not None
    return request.param


def _inputs(tokens=20):
    codes, scales = real_layer(64, 32, 8, 1)
    x = torch.randn((tokens, 64), generator=gen(2), device="cuda").bfloat16()
    bias = torch.randn(32, generator=gen(3), device="cuda")
    res = torch.randn((tokens, 32), generator=gen(4), device="cuda").bfloat16()
    return x, codes, scales, bias, res


def test_inputs_that_require_a_gradient_are_refused(path):
    x, codes, scales, bias, res = _inputs()
    want = sq.squant_linear(x, codes, scales, bias, residual=res)
    n = sq.squant_launch_count()
    for t in (x, scales, bias, res):
        t.requires_grad_()
        with pytest.raises(ValueError, match="autograd"):
            sq.squant_linear(x, codes, scales, bias, residual=res)
        t.requires_grad_(False)
    with pytest.raises(ValueError, match="autograd"):
        sq.squant_linear(x, codes, scales, bias, out=torch.empty_like(res).requires_grad_())
    with pytest.raises(ValueError, match="autograd"):
        sq.squant_linear_backward(res.detach().clone().requires_grad_(), codes, scales)
    assert sq.squant_launch_count() == n
    for t in (x, scales, bias, res):
        t.requires_grad_()
    with torch.no_grad():
        y = sq.squant_linear(x, codes, scales, bias, residual=res)
    assert same_bits(y, want) and not y.requires_grad
    # gradients into a parameter's own field: nothing to record
    g = sq.squant_linear_backward(res.detach(), codes, scales, bias, dbias=True)
    assert g.dx.shape == x.shape and not g.dx.requires_grad


def test_a_written_tensor_s_version(path):
    """Autograd must see that `out` has changed: a product that has kept it refuses its backward pass."""
    x, codes, scales, bias, res = _inputs()
    out = torch.ones_like(res)
    view = out[:, :16]
    weight = torch.ones_like(res, requires_grad=True)
    loss = (weight * out).sum()
    before = out._version
    assert sq.squant_linear(x, codes, scales, bias, out=out) is out
    assert out._version > before and view._version == out._version
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    before = out._version
    sq.squant_linear(x, codes, scales, bias)
    assert out._version == before
    with torch.inference_mode():   # such tensors have no version
        got = sq.squant_linear(x, codes, scales, bias, out=torch.empty_like(res))
        assert got.is_inference() and same_bits(got, out)


class Layer(torch.autograd.Function):
    """A layer whose codes stand for `weight` (a gradient for the weights) and whose activations are kept in 8 bits."""

    @staticmethod
    def forward(ctx, x, weight, bias, codes, scales, act, packed):
        y, z = sq.squant_linear(x, codes, scales, bias, act=act, pack_int4=packed, checkpoint=True)
        ctx.kept = codes, scales, bias, z, sq.squant_checkpoint(x), act, packed
        return y

    @staticmethod
    def backward(ctx, dy):
        codes, scales, bias, z, x, act, packed = ctx.kept
        g = sq.squant_linear_backward(dy.contiguous(), codes, scales, bias, cin=x.features, act=act, pack_int4=packed, z=z, x=x, dweight=True, dbias=True)
        return g.dx, g.dweight.float(), g.dbias, None, None, None, None


@pytest.mark.parametrize("tokens", [5, 70, 300])
def test_a_function_around_the_calls(path, tokens):
    x, codes, scales, bias, res = _inputs(tokens)
    codes = codes.clamp(-8, 7)
    stored = pack(codes)
    weight = (codes.float() * scales[:, None]).requires_grad_()
    x.requires_grad_()
    bias.requires_grad_()
    y = Layer.apply(x, weight, bias, stored, scales, "gelu", True)
    (y.float() * res.float()).sum().backward()
    with torch.no_grad():
        want, z = sq.squant_linear(x, stored, scales, bias, act="gelu", pack_int4=True, checkpoint=True)
        g = sq.squant_linear_backward(res, stored, scales, bias, cin=64, act="gelu", pack_int4=True, z=z, x=sq.squant_checkpoint(x), dweight=True, dbias=True)
    assert same_bits(y.detach(), want)
    assert same_bits(x.grad, g.dx) and same_bits(weight.grad, g.dweight.float()) and same_bits(bias.grad, g.dbias)
