"""Arguments of the linear operators: what the library refuses before any CUDA call (no GPU needed)."""
import ctypes

import pytest
import torch

import paper_2202_07471_b200 as sq
from paper_2202_07471_b200 import binding, linear

OK_PTR, ODD_PTR = 1 << 20, (1 << 20) + 1   # never dereferenced


def forward(**kw):
    a = linear.LinearArgs(tokens=4, cin=64, cout=32, dtype=0, act=0, flags=0, x=OK_PTR, x_stride=64, codes=OK_PTR, scales=OK_PTR, bias=None,
                          residual=None, residual_stride=0, y=OK_PTR, y_stride=32)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def backward(**kw):
    a = linear.LinearGradArgs(tokens=4, cin=64, cout=32, act=0, flags=0, dy=OK_PTR, dy_stride=32, codes=OK_PTR, scales=OK_PTR, dx=OK_PTR, dx_stride=64)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


CK = linear.CheckpointData(OK_PTR, OK_PTR)


@pytest.mark.parametrize("kw,code", [
    ({"tokens": -1}, -2), ({"tokens": (1 << 30) + 1}, -2), ({"cin": 0}, -2), ({"cout": -3}, -2), ({"cin": 1 << 30, "cout": 1 << 30, "x_stride": 1 << 30}, -2),
    ({"x_stride": 63}, -2), ({"y_stride": 31}, -2), ({"residual": OK_PTR, "residual_stride": 31}, -2), ({"x_stride": 0}, -2), ({"x_stride": -64}, -2),
    ({"dtype": 2}, -4), ({"act": 4}, -4), ({"flags": 1}, -4), ({"flags": 4}, -4),
    ({"x": None}, -1), ({"y": None}, -1), ({"codes": None}, -1), ({"scales": None}, -1), ({"z": linear.CheckpointData(OK_PTR, None)}, -1),
    ({"x": ODD_PTR}, -5), ({"y": ODD_PTR}, -5), ({"residual": ODD_PTR, "residual_stride": 32}, -5), ({"scales": OK_PTR + 2}, -5), ({"bias": OK_PTR + 2}, -5),
    ({"z": linear.CheckpointData(OK_PTR + 8, OK_PTR)}, -5), ({"z": linear.CheckpointData(OK_PTR, OK_PTR + 4)}, -5),
    ({"tokens": 40, "x_stride": 65}, -12), ({"tokens": 300}, -12), ({"tokens": 300, "workspace": OK_PTR, "workspace_bytes": 32 * 64 * 2 - 1}, -12),
    ({"tokens": 300, "workspace": OK_PTR + 8, "workspace_bytes": 1 << 30}, -12),
])
def test_forward_refuses(kw, code):
    lib = linear._lib()
    a = forward(**kw)
    assert lib.squant_linear(ctypes.byref(a), None) == code
    if code != -12:
        assert lib.squant_linear_workspace(ctypes.byref(a)) == code


@pytest.mark.parametrize("kw,code", [
    ({"tokens": -1}, -2), ({"cin": 0}, -2), ({"cout": 0}, -2), ({"dy_stride": 31}, -2), ({"dx_stride": 63}, -2),
    ({"dweight": OK_PTR, "dweight_stride": 63, "x": CK}, -2), ({"act": 4}, -4), ({"flags": 1}, -4),
    ({"dy": None}, -1), ({"codes": None}, -1), ({"scales": None}, -1), ({"act": 1}, -1), ({"dscales": OK_PTR}, -1),
    ({"dx": None, "codes": None, "scales": None, "dscales": OK_PTR, "z": CK}, -1), ({"dweight": OK_PTR, "dweight_stride": 64}, -1),
    ({"dy": ODD_PTR}, -5), ({"dx": ODD_PTR}, -5), ({"dbias": OK_PTR + 2}, -5), ({"z": linear.CheckpointData(OK_PTR + 1, OK_PTR)}, -5),
    ({}, -12), ({"workspace": OK_PTR, "workspace_bytes": 4 * 32 * 2 - 1}, -12), ({"workspace": OK_PTR + 2, "workspace_bytes": 1 << 20}, -12),
])
def test_backward_refuses(kw, code):
    lib = linear._lib()
    a = backward(**kw)
    assert lib.squant_linear_backward(ctypes.byref(a), None) == code
    if code != -12:
        assert lib.squant_linear_backward_workspace(ctypes.byref(a)) == code


def test_null_arguments():
    lib = linear._lib()
    assert lib.squant_linear(None, None) == -1 and lib.squant_linear_workspace(None) == -1
    assert lib.squant_linear_backward(None, None) == -1 and lib.squant_linear_backward_workspace(None) == -1
    none = linear.CheckpointData(None, None)
    assert lib.squant_checkpoint(OK_PTR, 3, 40, 40, None, None) == -1
    assert lib.squant_checkpoint(OK_PTR, 3, 40, 40, ctypes.byref(none), None) == -1
    assert lib.squant_checkpoint(None, 3, 40, 40, ctypes.byref(CK), None) == -1
    assert lib.squant_checkpoint(OK_PTR, 3, 0, 40, ctypes.byref(CK), None) == -2
    assert lib.squant_checkpoint(OK_PTR, -1, 40, 40, ctypes.byref(CK), None) == -2
    assert lib.squant_checkpoint(OK_PTR, 3, 40, 39, ctypes.byref(CK), None) == -2
    assert lib.squant_checkpoint(ODD_PTR, 3, 40, 40, ctypes.byref(CK), None) == -5
    assert lib.squant_checkpoint_restore(None, 3, 40, OK_PTR, 40, None) == -1
    assert lib.squant_checkpoint_restore(ctypes.byref(CK), 3, 40, None, 40, None) == -1
    assert lib.squant_checkpoint_restore(ctypes.byref(CK), 3, 40, OK_PTR, 39, None) == -2
    assert lib.squant_checkpoint_restore(ctypes.byref(linear.CheckpointData(OK_PTR + 8, OK_PTR)), 3, 40, OK_PTR, 40, None) == -5
    assert "workspace" in lib.squant_strerror(-12).decode()


def test_calls_without_tokens_need_nothing():
    lib = linear._lib()
    a = forward(tokens=0, x=None, y=None)
    assert lib.squant_linear_workspace(ctypes.byref(a)) == 0 and lib.squant_linear(ctypes.byref(a), None) == 0
    b = backward(tokens=0, dy=None, dx=OK_PTR)
    assert lib.squant_linear_backward_workspace(ctypes.byref(b)) == 0
    assert lib.squant_checkpoint(None, 0, 40, 40, ctypes.byref(CK), None) == 0
    assert lib.squant_checkpoint_restore(ctypes.byref(CK), 0, 40, None, 40, None) == 0


def test_workspace_sizes():
    """What the header documents: nothing for rows on 16 bytes up to 256 tokens; copies of x and of the codes, the codes as 16-bit floats,
    dz and dz * s."""
    lib = linear._lib()
    need = lambda **kw: lib.squant_linear_workspace(ctypes.byref(forward(**kw)))
    assert need() == 0 and need(tokens=256) == 0 and need(tokens=8, x=OK_PTR + 2) == 0
    assert need(tokens=9, x=OK_PTR + 2) == 9 * 64 * 2                      # rows that start anywhere
    assert need(tokens=9, cin=61, x_stride=61) == 9 * 64 * 2 + 32 * 64     # and the codes'
    assert need(tokens=257) == 32 * 64 * 2
    assert need(tokens=257, cin=61, x_stride=61) == 257 * 64 * 2 + 32 * 64 * 2
    need = lambda **kw: lib.squant_linear_backward_workspace(ctypes.byref(backward(**kw)))
    assert need() == 4 * 32 * 2
    assert need(act=1, z=CK, dx=None) == 0                                 # nothing asked for
    assert need(act=1, z=CK, dx=None, dweight=OK_PTR, dweight_stride=64, x=CK) == 4 * 32 * 2 + 4 * 64 * 2
    assert need(dx=None, dweight=OK_PTR, dweight_stride=64, x=CK) == 4 * 64 * 2   # dz is dy itself
    assert need(tokens=1000) == 1000 * 32 * 2 + 32 * 64 * 2
    assert need(cin=61, dx_stride=61) == 4 * 32 * 2 + 32 * 64


def test_workspace_of_long_contractions():
    """More than 65,536 terms go in parts, whose fp32 sums [rows][columns rounded up to 32] lie behind the rest; up to 256 tokens eight thread
    blocks or warps share 524,288."""
    lib = linear._lib()
    need = lambda **kw: lib.squant_linear_workspace(ctypes.byref(forward(**kw)))
    k = 1 << 16
    assert need(tokens=300, cin=k, x_stride=k) == 32 * k * 2
    assert need(tokens=300, cin=k + 16, x_stride=k + 16) == 32 * (k + 16) * 2 + 300 * 32 * 4
    assert need(tokens=300, cin=k + 16, x_stride=k + 16, cout=33, y_stride=33) == 33 * (k + 16) * 2 + 300 * 64 * 4
    assert need(tokens=4, cin=8 * k, x_stride=8 * k) == 0 and need(tokens=40, cin=8 * k, x_stride=8 * k) == 0
    for tokens in (1, 4, 40):
        assert need(tokens=tokens, cin=8 * k + 16, x_stride=8 * k + 16) == 32 * (8 * k + 16) * 2 + tokens * 32 * 4
    need = lambda **kw: lib.squant_linear_backward_workspace(ctypes.byref(backward(**kw)))
    assert need(tokens=k, dx=None, dweight=OK_PTR, dweight_stride=64, x=CK) == k * 64 * 2
    assert need(tokens=k + 1, dx=None, dweight=OK_PTR, dweight_stride=64, x=CK) == (k + 1) * 64 * 2 + 32 * 64 * 4
    assert need(tokens=300, cout=k + 8, dy_stride=k + 8) == 300 * (k + 8) * 2 + (k + 8) * 64 * 2 + 300 * 64 * 4
    assert need(tokens=4, cout=8 * k, dy_stride=8 * k) == 4 * 8 * k * 2
    assert need(tokens=4, cout=8 * k + 8, dy_stride=8 * k + 8) == 4 * (8 * k + 8) * 2 + (8 * k + 8) * 64 * 2 + 4 * 64 * 4
    # both sums take the same place
    assert need(tokens=k + 1, cout=k + 8, dy_stride=k + 8, dweight=OK_PTR, dweight_stride=64, x=CK) == (k + 1) * (k + 8) * 2 + (k + 8) * 64 * 2 + (k + 8) * 64 * 4


FEW, FUSED, DENSE, WIDE = 1, 2, 3, 4


@pytest.mark.parametrize("kw,kernel", [
    ({"tokens": 0}, 0), ({"tokens": 1}, FEW), ({"tokens": 8}, FEW), ({"tokens": 9}, FEW), ({"tokens": 256}, FEW), ({"tokens": 257}, DENSE),
    ({"tokens": 8, "z": CK}, FUSED), ({"tokens": 256, "z": CK}, FUSED), ({"tokens": 257, "z": CK}, DENSE), ({"tokens": 9, "x": OK_PTR + 2}, FUSED),
    ({"tokens": 9, "x": OK_PTR + 16}, FUSED), ({"tokens": 9, "x_stride": 72}, FUSED), ({"tokens": 9, "cin": 61, "x_stride": 61}, FUSED),
    ({"tokens": 16, "cin": 4096, "x_stride": 4096, "cout": 12288, "y_stride": 12288}, FEW), ({"tokens": 16, "cin": 4096, "x_stride": 4096, "cout": 12289, "y_stride": 12289}, FUSED),
    ({"tokens": 2100, "cout": 1700, "y_stride": 1700}, WIDE), ({"tokens": 2100, "cout": 2100, "y_stride": 2100}, DENSE),
    ({"tokens": 5, "cin": 1 << 19, "x_stride": 1 << 19}, FEW), ({"tokens": 5, "cin": (1 << 19) + 16, "x_stride": (1 << 19) + 16}, DENSE),
    # up to eight tokens: rows of x, of the codes or both off 16 bytes, either side of the line for them
    ({"tokens": 8, "cin": 4096, "x_stride": 4096, "cout": 4096, "y_stride": 4096}, FEW), ({"tokens": 8, "cin": 4096, "x_stride": 4104, "cout": 4096, "y_stride": 4096}, FEW),
    ({"tokens": 8, "cin": 2048, "x_stride": 2049, "cout": 4096, "y_stride": 4096}, FEW), ({"tokens": 8, "cin": 2049, "x_stride": 2049, "cout": 4096, "y_stride": 4096}, FUSED),
    ({"tokens": 1, "cin": 4096, "x_stride": 4097, "cout": 4096, "y_stride": 4096}, FEW), ({"tokens": 2, "cin": 4096, "x_stride": 4097, "cout": 4096, "y_stride": 4096}, FUSED),
    ({"tokens": 1, "x": OK_PTR + 2, "cin": 4096, "x_stride": 4096, "cout": 256, "y_stride": 256}, FUSED), ({"tokens": 1, "x": OK_PTR + 2, "cin": 2000, "x_stride": 2000, "cout": 256, "y_stride": 256}, FEW),
    ({"tokens": -1}, -2), ({"x": None}, -1), ({"act": 9}, -4), ({"x": ODD_PTR}, -5)])
def test_which_kernel_a_call_takes(kw, kernel):
    assert linear._lib().squant_linear_plan(ctypes.byref(forward(**kw))) == kernel


def test_tensors_have_to_be_on_a_gpu():
    x, codes, scales = torch.zeros(2, 64, dtype=torch.bfloat16), torch.zeros(32, 64, dtype=torch.int8), torch.ones(32)
    with pytest.raises(ValueError, match="CUDA"):
        sq.squant_linear(x, codes, scales)
    with pytest.raises(ValueError, match="CUDA"):
        sq.squant_linear_backward(torch.zeros(2, 32, dtype=torch.bfloat16), codes, scales)
    with pytest.raises(ValueError, match="CUDA"):
        sq.squant_checkpoint(x)
    with pytest.raises(ValueError, match="CUDA"):
        sq.squant_checkpoint_restore(sq.Checkpoint(torch.zeros(2, 64, dtype=torch.int8), torch.zeros(2, 2, dtype=torch.uint8), 64))


def test_the_extension_has_the_library_s_structs():
    m = binding._marshal
    if m is None:
        pytest.skip("the descriptor extension is not built")
    assert m.linear_bytes == ctypes.sizeof(linear.LinearArgs) and m.linear_grad_bytes == ctypes.sizeof(linear.LinearGradArgs)


def test_inputs_that_require_a_gradient_are_refused():
    """The calls are not recorded by autograd: a loss on their results would train nothing that lies before them."""
    x, codes, scales = torch.zeros(2, 64, dtype=torch.bfloat16), torch.zeros(32, 64, dtype=torch.int8), torch.ones(32)
    bias, res, dy = torch.zeros(32), torch.zeros(2, 32, dtype=torch.bfloat16), torch.zeros(2, 32, dtype=torch.bfloat16)
    for t in (x, scales, bias, res):
        t.requires_grad_()
        with pytest.raises(ValueError, match="autograd"):
            sq.squant_linear(x, codes, scales, bias, residual=res)
        with torch.no_grad(), pytest.raises(ValueError, match="CUDA"):   # goes on to the next check
            sq.squant_linear(x, codes, scales, bias, residual=res)
        t.requires_grad_(False)
    with pytest.raises(ValueError, match="autograd"):
        sq.squant_linear(x, codes, scales, out=res.requires_grad_())
    with pytest.raises(ValueError, match="autograd"):
        sq.squant_linear_backward(dy.requires_grad_(), codes, scales)
