"""Linear layers on quantized weights and 8-bit activation checkpoints: binding of the squant_linear* and
squant_checkpoint* entry points (argument marshalling only; all work runs in the CUDA library).

Activations are bfloat16 or float16 tensors [..., features]; leading dimensions count as tokens.  Codes and scales are
what squant_quantize_layer / squant_quantize_model wrote for a layer of weights [cout, cin]: int8 codes [cout, cin], or
[cout, ceil(cin / 2)] with pack_int4.  Outputs are allocated from PyTorch's caching allocator on the current stream, or on
`stream` where one is given.

None of the calls is recorded by autograd.  squant_linear refuses inputs that require a gradient where one would be recorded (grad mode on), and
squant_linear_backward a dy that does; a torch.autograd.Function around the calls, in whose forward and backward grad mode is off, makes
them part of a graph.
"""
from __future__ import annotations

import ctypes
import math
from dataclasses import dataclass
from typing import Optional

import torch

from . import binding
from .binding import FLAG_PACK_INT4, _check, load_library

ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}
_TYPES = {torch.bfloat16: 0, torch.float16: 1}

GROUP = 32   # features that share an exponent in a checkpoint


class CheckpointData(ctypes.Structure):
    _fields_ = [("codes", ctypes.c_void_p), ("exps", ctypes.c_void_p)]


class LinearArgs(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_int64), ("cin", ctypes.c_int32), ("cout", ctypes.c_int32), ("dtype", ctypes.c_uint32),
                ("act", ctypes.c_uint32), ("flags", ctypes.c_uint32), ("x", ctypes.c_void_p), ("x_stride", ctypes.c_int64),
                ("codes", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("bias", ctypes.c_void_p), ("residual", ctypes.c_void_p),
                ("residual_stride", ctypes.c_int64), ("y", ctypes.c_void_p), ("y_stride", ctypes.c_int64), ("z", CheckpointData),
                ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_int64)]


class LinearGradArgs(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_int64), ("cin", ctypes.c_int32), ("cout", ctypes.c_int32), ("act", ctypes.c_uint32),
                ("flags", ctypes.c_uint32), ("dy", ctypes.c_void_p), ("dy_stride", ctypes.c_int64), ("codes", ctypes.c_void_p),
                ("scales", ctypes.c_void_p), ("bias", ctypes.c_void_p), ("z", CheckpointData), ("x", CheckpointData),
                ("dx", ctypes.c_void_p), ("dx_stride", ctypes.c_int64), ("dweight", ctypes.c_void_p), ("dweight_stride", ctypes.c_int64),
                ("dbias", ctypes.c_void_p), ("dscales", ctypes.c_void_p), ("workspace", ctypes.c_void_p),
                ("workspace_bytes", ctypes.c_int64)]


@dataclass
class Checkpoint:
    """An activation [rows, features] in 8 bits: int8 codes [rows, features rounded up to 32] and uint8 exponents
    [rows, groups of 32], both contiguous and on 16 bytes; the values are codes * 2^(exponent - 127)."""
    codes: torch.Tensor
    exps: torch.Tensor
    features: int


@dataclass
class LinearGrads:
    """Gradients of a linear layer, None where not asked for."""
    dx: Optional[torch.Tensor] = None        # bfloat16 [..., cin], leading dimensions as dy's
    dweight: Optional[torch.Tensor] = None   # bfloat16 [cout, cin], of the weights codes * scales
    dbias: Optional[torch.Tensor] = None     # fp32 [cout]
    dscales: Optional[torch.Tensor] = None   # fp32 [cout]


_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device   # the latter also initializes CUDA
_ready = None
_address = {}   # of the library's functions, for the native extension


def _lib() -> ctypes.CDLL:
    global _ready
    lib = load_library()
    if _ready is not lib:
        vp, i64, ck = ctypes.c_void_p, ctypes.c_int64, ctypes.POINTER(CheckpointData)
        lib.squant_checkpoint.argtypes = [vp, i64, ctypes.c_int32, i64, ck, vp]
        lib.squant_checkpoint_restore.argtypes = [ck, i64, ctypes.c_int32, vp, i64, vp]
        lib.squant_linear.argtypes = [ctypes.POINTER(LinearArgs), vp]
        lib.squant_linear_workspace.argtypes = [ctypes.POINTER(LinearArgs)]
        lib.squant_linear_plan.argtypes = [ctypes.POINTER(LinearArgs)]
        lib.squant_linear_backward.argtypes = [ctypes.POINTER(LinearGradArgs), vp]
        lib.squant_linear_backward_workspace.argtypes = [ctypes.POINTER(LinearGradArgs)]
        for f in ("squant_checkpoint", "squant_checkpoint_restore", "squant_linear", "squant_linear_plan", "squant_linear_backward"):
            getattr(lib, f).restype = ctypes.c_int
        for f in ("squant_linear_workspace", "squant_linear_backward_workspace"):
            getattr(lib, f).restype = i64
        for f in ("squant_checkpoint", "squant_checkpoint_restore", "squant_linear", "squant_linear_workspace", "squant_linear_backward",
                  "squant_linear_backward_workspace"):
            _address[f] = ctypes.cast(getattr(lib, f), ctypes.c_void_p).value
        _ready = lib
    return lib


_checked = (None, None, None)   # extension, library, and the extension if it was built with the library's argument structs


def _native():
    """The extension that makes whole calls for plain tensors (None: not built, or built with other argument structs)."""
    global _checked
    if _checked[0] is binding._marshal and _checked[1] is binding._lib and _checked[1] is not None:
        return _checked[2]
    if not torch.cuda.is_initialized():
        return None
    m, lib = binding._marshal, _lib()
    fits = (getattr(m, "linear_bytes", None) == ctypes.sizeof(LinearArgs) and getattr(m, "linear_grad_bytes", None) == ctypes.sizeof(LinearGradArgs)
            and binding._raw_stream is not None)
    if fits:
        m.use(_address["squant_linear"], _address["squant_linear_workspace"], _address["squant_linear_backward"],
              _address["squant_linear_backward_workspace"], _address["squant_checkpoint"], _address["squant_checkpoint_restore"])
    _checked = (m, lib, m if fits else None)
    return _checked[2]


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _result(got):
    """What the extension returned, if it is not an error code."""
    if type(got) is int:
        _check(got)
    return got


class _On:
    """The tensors' device current and, where a stream is given, that stream too, so that what is allocated here
    belongs to the stream that the kernels run on."""

    def __init__(self, device: torch.device, stream: Optional[torch.cuda.Stream]):
        if device.type != "cuda":
            raise ValueError("the linear operators need CUDA tensors")
        if stream is not None and stream.device != device:
            raise ValueError(f"the stream belongs to {stream.device}, the tensors to {device}")
        self.guards = []
        if stream is not None:
            self.guards.append(torch.cuda.stream(stream))
        elif device.index != torch.cuda.current_device():
            self.guards.append(torch.cuda.device(device))

    def __enter__(self) -> ctypes.c_void_p:
        for g in self.guards:
            g.__enter__()
        return binding._stream_handle(None)

    def __exit__(self, *exc):
        for g in reversed(self.guards):
            g.__exit__(*exc)


def _no_graph(what: str, *inputs: Optional[torch.Tensor]) -> None:
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in inputs):
        raise ValueError(f"{what} is not recorded by autograd: call it under torch.no_grad(), or from the forward and backward of a torch.autograd.Function, "
                         "with squant_linear_backward for the gradients")


def _rows(t: torch.Tensor, what: str) -> torch.Tensor:
    """[..., features] as [tokens, features] without a copy."""
    if t.dim() == 0 or t.shape[-1] == 0:
        raise ValueError(f"{what} must be a tensor [..., features]")
    if t.dim() != 2:
        try:
            t = t.view(math.prod(t.shape[:-1]), t.shape[-1])
        except RuntimeError:
            raise ValueError(f"the leading dimensions of {what} cannot be seen as rows without a copy") from None
    if t.shape[1] > 1 and t.stride(1) != 1:
        raise ValueError(f"the features of {what} must lie next to each other")
    return t


def _vector(t: Optional[torch.Tensor], n: int, what: str, device: torch.device) -> Optional[torch.Tensor]:
    if t is None:
        return None
    if t.dtype != torch.float32 or t.shape != (n,) or not t.is_contiguous() or t.device != device:
        raise ValueError(f"{what} must be a contiguous fp32 tensor [{n}] next to the activations")
    return t


def _codes(codes: torch.Tensor, cin: int, pack_int4: bool, device: torch.device) -> int:
    """Number of output channels."""
    width = (cin + 1) // 2 if pack_int4 else cin
    if codes.dtype != torch.int8 or not codes.is_contiguous() or codes.device != device or codes.dim() < 2 or math.prod(codes.shape[1:]) != width:
        raise ValueError(f"codes must be a contiguous int8 tensor [cout, {width}] next to the activations")
    return int(codes.shape[0])


def _act(act: str) -> int:
    if act not in ACTIVATIONS:
        raise ValueError(f"unknown activation {act!r}: one of {', '.join(ACTIVATIONS)}")
    return ACTIVATIONS[act]


def _checkpoint_data(c: Optional[Checkpoint], rows: int, features: int, what: str, device: torch.device) -> CheckpointData:
    if c is None:
        return CheckpointData(None, None)
    groups = -(-features // GROUP)
    if (c.features != features or c.codes.dtype != torch.int8 or c.exps.dtype != torch.uint8 or c.codes.shape != (rows, groups * GROUP)
            or c.exps.shape != (rows, groups) or not c.codes.is_contiguous() or not c.exps.is_contiguous()
            or c.codes.device != device or c.exps.device != device):
        raise ValueError(f"{what} must be a Checkpoint of [{rows}, {features}] next to the other tensors")
    return CheckpointData(_ptr(c.codes), _ptr(c.exps))


def _new_checkpoint(rows: int, features: int, device: torch.device) -> Checkpoint:
    groups = -(-features // GROUP)
    return Checkpoint(torch.empty((rows, groups * GROUP), dtype=torch.int8, device=device),
                      torch.empty((rows, groups), dtype=torch.uint8, device=device), features)


def _run(fn, need, args, handle, device: torch.device) -> None:
    """The call with the workspace it needs (and its argument checks, which the size comes with)."""
    size = need(ctypes.byref(args))
    if size < 0:
        _check(int(size))
    if size:
        workspace = torch.empty(size, dtype=torch.uint8, device=device)
        args.workspace, args.workspace_bytes = workspace.data_ptr(), size
    _check(fn(ctypes.byref(args), handle))


def squant_checkpoint(x: torch.Tensor, stream: Optional[torch.cuda.Stream] = None) -> Checkpoint:
    """An activation (bfloat16 [..., features]) in 8 bits: 33/64 of its bytes, at most half a step of the largest of 32
    neighbours off (2^-7 of its power of two).  The checkpoint and what is restored from it carry no gradient."""
    native = None if stream is not None else _native()
    if native is not None:
        device = _device()
        got = native.checkpoint(binding._raw_stream(device), device, x)
        if got is not None:
            return Checkpoint(*_result(got))
    with _On(x.device, stream) as handle:
        if x.dtype != torch.bfloat16:
            raise ValueError("checkpoints are taken of bfloat16 tensors")
        x = _rows(x, "x")
        c = _new_checkpoint(x.shape[0], x.shape[1], x.device)
        _check(_lib().squant_checkpoint(_ptr(x), x.shape[0], x.shape[1], x.stride(0), ctypes.byref(CheckpointData(_ptr(c.codes), _ptr(c.exps))), handle))
    return c


def squant_checkpoint_restore(c: Checkpoint, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """The values of a checkpoint as a bfloat16 tensor [rows, features], exactly."""
    native = None if stream is not None else _native()
    if native is not None:
        device = _device()
        got = native.restore(binding._raw_stream(device), device, c.codes, c.exps, c.features)
        if got is not None:
            return _result(got)
    device = c.codes.device
    with _On(device, stream) as handle:
        rows = c.codes.shape[0]
        data = _checkpoint_data(c, rows, c.features, "c", device)
        out = torch.empty((rows, c.features), dtype=torch.bfloat16, device=device)
        _check(_lib().squant_checkpoint_restore(ctypes.byref(data), rows, c.features, _ptr(out), c.features, handle))
    return out


def squant_linear(x: torch.Tensor, codes: torch.Tensor, scales: torch.Tensor, bias: Optional[torch.Tensor] = None, *,
                  residual: Optional[torch.Tensor] = None, act: str = "none", pack_int4: bool = False, checkpoint: bool = False,
                  out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None):
    """act((x @ codes^T) * scales + bias) + residual, in the type of x (bfloat16 or float16), [..., cout].

    bias: fp32 [cout]; residual: like the output.  act: "none", "relu", "gelu" (with erf) or "silu".  With `checkpoint`
    returns (y, Checkpoint of the pre-activation [tokens, cout]) for squant_linear_backward.  out: the tensor to write; it may
    be `residual` itself, and must not overlap the other inputs otherwise."""
    native = None if stream is not None else _native()
    if native is not None:
        device = _device()
        got = native.linear(binding._raw_stream(device), device, x, codes, scales, bias, residual, out, ACTIVATIONS.get(act, -1), pack_int4, checkpoint)
        if got is not None:
            got = _result(got)
            return (got[0], Checkpoint(got[1], got[2], codes.shape[0])) if checkpoint else got
    _no_graph("squant_linear", x, scales, bias, residual, out)
    written = out
    device = x.device
    with _On(device, stream) as handle:
        if x.dtype not in _TYPES:
            raise ValueError("activations must be bfloat16 or float16")
        shape = x.shape[:-1]
        x = _rows(x, "x")
        tokens, cin = x.shape
        cout = _codes(codes, cin, pack_int4, device)
        _vector(scales, cout, "scales", device)
        _vector(bias, cout, "bias", device)
        if out is None:
            out = torch.empty((*shape, cout), dtype=x.dtype, device=device)
        for name, t in (("residual", residual), ("out", out)):
            if t is not None and (t.dtype != x.dtype or t.shape != (*shape, cout) or t.device != device):
                raise ValueError(f"{name} must be a {x.dtype} tensor {[*shape, cout]} next to the activations")
        y = _rows(out, "out")
        r = None if residual is None else _rows(residual, "residual")
        z = _new_checkpoint(tokens, cout, device) if checkpoint else None
        a = LinearArgs(tokens, cin, cout, _TYPES[x.dtype], _act(act), FLAG_PACK_INT4 if pack_int4 else 0, _ptr(x), x.stride(0),
                       _ptr(codes), _ptr(scales), _ptr(bias), _ptr(r), 0 if r is None else r.stride(0), _ptr(y), y.stride(0),
                       CheckpointData(_ptr(z.codes), _ptr(z.exps)) if z else CheckpointData(None, None), None, 0)
        lib = _lib()
        _run(lib.squant_linear, lib.squant_linear_workspace, a, handle, device)
    if written is not None and not written.is_inference():
        torch.autograd.graph.increment_version(written)
    return (out, z) if checkpoint else out


def squant_linear_backward(dy: torch.Tensor, codes: torch.Tensor, scales: torch.Tensor, bias: Optional[torch.Tensor] = None, *,
                           cin: Optional[int] = None, act: str = "none", pack_int4: bool = False, z: Optional[Checkpoint] = None,
                           x: Optional[Checkpoint] = None, dx: bool = True, dweight: bool = False, dbias: bool = False,
                           dscales: bool = False, stream: Optional[torch.cuda.Stream] = None) -> LinearGrads:
    """Gradients of squant_linear's output act((x @ codes^T) * scales + bias) for dy (bfloat16 [..., cout]).

    z: checkpoint of the pre-activation (needed with an activation and for dscales); x: checkpoint of the input (needed
    for dweight); cin is needed with pack_int4, whose rows do not tell it.  dweight is the gradient of the weights
    codes * scales: a training loop applies it to the weights that it quantizes.

    dscales divides (z's checkpoint - bias) by the scales, which must not be 0, and with it the checkpoint's step, which the largest of 32 neighbouring channels
    sets: 0.9 % off the layer's own gradient for channels of one size, 8 to 20 % where their sizes spread as exp(N(0, 1)), of no use where some are
    tens of times smaller than their neighbours.  There, ask for dweight and take (dweight.float() * codes).sum(1): the same gradient from the input,
    0.9 % off at any spread without an activation (its slope is read from z's checkpoint too)."""
    native = None if stream is not None else _native()
    if native is not None and dy.dim() and (z is None or z.features == dy.shape[-1]) and not (cin is None and pack_int4):
        device = _device()
        width = math.prod(codes.shape[1:]) if cin is None else cin
        if x is None or x.features == width:
            got = native.linear_backward(binding._raw_stream(device), device, dy, codes, scales, bias, z and z.codes, z and z.exps, x and x.codes,
                                         x and x.exps, width, ACTIVATIONS.get(act, -1), pack_int4, dx, dweight, dbias, dscales)
            if got is not None:
                return LinearGrads(*_result(got))
    _no_graph("squant_linear_backward", dy)
    device = dy.device
    with _On(device, stream) as handle:
        if dy.dtype != torch.bfloat16:
            raise ValueError("gradients are bfloat16 tensors")
        shape = dy.shape[:-1]
        d = _rows(dy, "dy")
        tokens, cout = d.shape
        if cin is None:
            if pack_int4:
                raise ValueError("cin must be given with pack_int4")
            cin = math.prod(codes.shape[1:])
        if _codes(codes, cin, pack_int4, device) != cout:
            raise ValueError(f"codes have {codes.shape[0]} output channels, dy {cout}")
        _vector(scales, cout, "scales", device)
        _vector(bias, cout, "bias", device)
        number = _act(act)
        zd = _checkpoint_data(z, tokens, cout, "z", device)
        xd = _checkpoint_data(x, tokens, cin, "x", device)
        if z is None and (number or dscales):
            raise ValueError("z, the checkpoint of the pre-activation, is needed with an activation and for dscales")
        if x is None and dweight:
            raise ValueError("x, the checkpoint of the input, is needed for dweight")
        bf16, f32 = dict(dtype=torch.bfloat16, device=device), dict(dtype=torch.float32, device=device)
        g = LinearGrads(torch.empty((*shape, cin), **bf16) if dx else None, torch.empty((cout, cin), **bf16) if dweight else None,
                        torch.empty(cout, **f32) if dbias else None, torch.empty(cout, **f32) if dscales else None)
        a = LinearGradArgs(tokens, cin, cout, number, FLAG_PACK_INT4 if pack_int4 else 0, _ptr(d), d.stride(0), _ptr(codes), _ptr(scales),
                           _ptr(bias), zd, xd, _ptr(g.dx), cin, _ptr(g.dweight), cin, _ptr(g.dbias), _ptr(g.dscales), None, 0)
        lib = _lib()
        _run(lib.squant_linear_backward, lib.squant_linear_backward_workspace, a, handle, device)
    return g
