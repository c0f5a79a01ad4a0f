"""Inputs and 64-bit references of the linear operators' tests (plain torch; nothing of the library)."""
import math

import torch

GROUP = 32
ACTS = ("none", "relu", "gelu", "silu")


def gen(seed, device="cuda"):
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    return g


def padded(t, pad, fill=None):
    """`t` as a view of a wider buffer; the rest of the buffer holds `fill`.  Returns (view, buffer)."""
    buf = torch.empty((t.shape[0], t.shape[1] + pad), dtype=t.dtype, device=t.device)
    buf.fill_(float("nan") if fill is None else fill)
    buf[:, :t.shape[1]] = t
    return buf[:, :t.shape[1]], buf


def pack(codes):
    if codes.shape[1] % 2:   # the unused nibble of an odd row may hold anything
        codes = torch.cat((codes, torch.full_like(codes[:, :1], -3)), 1)
    u = codes.to(torch.int32)
    return ((u[:, 0::2] & 15) | ((u[:, 1::2] & 15) << 4)).to(torch.uint8).view(torch.int8).contiguous()


def int_layer(cin, cout, bits, seed, lowest=-6):
    """Codes over their whole range and scales that are powers of two."""
    g = gen(seed)
    lo, hi = (-8, 7) if bits == 4 else (-128, 127)
    codes = torch.randint(lo, hi + 1, (cout, cin), generator=g, device="cuda", dtype=torch.int32).to(torch.int8)
    scales = torch.exp2(torch.randint(lowest, 3, (cout,), generator=g, device="cuda").float())
    return codes, scales


def real_layer(cin, cout, bits, seed):
    g = gen(seed)
    qmax = 7 if bits == 4 else 127
    w = torch.randn((cout, cin), generator=g, device="cuda") / math.sqrt(cin)
    scales = (w.abs().amax(1) / qmax).clamp(min=1e-6)
    return torch.clamp(torch.round(w / scales[:, None]), -qmax, qmax).to(torch.int8), scales


def act64(z, act):
    if act == "relu":
        return torch.clamp(z, min=0.0)
    if act == "gelu":
        return z * 0.5 * torch.special.erfc(-z / math.sqrt(2.0))
    if act == "silu":
        return z * torch.sigmoid(z)
    return z


def slope64(z, act):
    if act == "relu":
        return (z > 0).double()
    if act == "gelu":
        return 0.5 * torch.special.erfc(-z / math.sqrt(2.0)) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    if act == "silu":
        p = torch.sigmoid(z)
        return p * (1.0 + z * (1.0 - p))
    return torch.ones_like(z)


def encode64(v):
    """The checkpoint's definition in 64 bits: int8 codes and exponents (no infinities or NaN)."""
    rows, n = v.shape
    full = torch.nn.functional.pad(v.double(), (0, -n % GROUP)).reshape(rows, -1, GROUP)
    a = full.abs().amax(2)
    top = torch.frexp(a).exponent - 1                     # floor(log2 a); 0 for a = 0, which the next line's zero replaces
    e = torch.where(a == 0, 1, torch.clamp(top + 127 - 6, min=1))
    q = torch.clamp(torch.round(torch.ldexp(full, (127 - e)[..., None])), -127, 127)
    return q.to(torch.int8).reshape(rows, -1), e.to(torch.uint8)


def decode64(codes, exps, n):
    v = torch.ldexp(codes.double().reshape(codes.shape[0], -1, GROUP), exps.to(torch.int32)[..., None] - 127)
    v = torch.where(exps[..., None] == 255, float("nan"), v)
    return v.reshape(codes.shape[0], -1)[:, :n]


def same_bits(a, b):
    kind = {2: torch.int16, 4: torch.int32, 1: torch.int8}[a.element_size()]
    return a.shape == b.shape and a.dtype == b.dtype and torch.equal(a.contiguous().view(kind), b.contiguous().view(kind))
