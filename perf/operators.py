"""The calls that the operators of a quantized linear layer are measured by.

A layer holds what the quantizer writes: int8 codes [cout, cin] (or packed int4, two codes a byte) and one fp32
scale per output channel.  Three operators:

  "linear"      y = act((x @ codes^T) * scales + bias) + residual, with or without a checkpoint of the
                pre-activation in 8 bits
  "checkpoint"  an activation into 8 bits (groups of 32 features with a power-of-two scale) and back
  "backward"    the layer's gradients from dy, the codes and the 8-bit checkpoints: dx, dbias, dscales, dweight

The layer sizes are those of `cases.py`'s linear layers (4096 to 4096, 4096 to 11008, 11008 to 4096, and
1537 to 1001, where no row starts on a vector) and smaller ones; tokens go from one to 8192.

Fields of a case:
  op         one of the above
  tokens, cin, cout
  dtype      "bf16" or "fp16" (x, residual, y); gradients and checkpoints are bf16
  bits       8: int8 codes, 4: packed int4 codes
  act        "none", "relu", "gelu" (erf), "silu"
  bias, residual, save (a checkpoint of the pre-activation is written too)
  pad        extra elements between the rows of x, residual and dy (they are views of wider buffers)
  want       gradients asked for, of "x", "w", "b", "s"
"""
import math

import torch

own = False

_GROUP = 32
_TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
_LINEAR = {"op": "linear", "dtype": "bf16", "bits": 4, "act": "none", "bias": False, "residual": False, "save": False, "pad": 0}
_CHECKPOINT = {"op": "checkpoint", "pad": 0}
_BACKWARD = {"op": "backward", "bits": 4, "act": "none", "want": "xwb", "pad": 0}


def _case(base, name=None, **kw):
    c = dict(base, **kw)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token of one sequence: latency and the bytes of the codes
        _case(_LINEAR, "decode_1", tokens=1, cin=4096, cout=4096, residual=True),
        # a batch of sequences, one token each, into the wide layer of a feed-forward block
        _case(_LINEAR, "decode_16", tokens=16, cin=4096, cout=11008, dtype="fp16", act="silu", bias=True),
        # a short prompt at an odd size: rows that start anywhere
        _case(_LINEAR, "linear_odd", tokens=77, cin=1537, cout=1001, bits=8, act="gelu", bias=True, residual=True, pad=3),
        # a training step's forward pass, which saves its pre-activation
        _case(_LINEAR, "linear_train", tokens=2048, cin=4096, cout=4096, bits=8, act="gelu", bias=True, save=True),
        # prompts: the large matrix product
        _case(_LINEAR, "linear_prompt", tokens=4096, cin=4096, cout=11008, residual=True, bias=True),
        # activations of a small batch into 8 bits and back
        _case(_CHECKPOINT, "checkpoint_small", tokens=48, cin=1001),
        # activations of a training step
        _case(_CHECKPOINT, "checkpoint_large", tokens=8192, cin=11008),
        # gradients of a small layer with few tokens (latency)
        _case(_BACKWARD, "backward_small", tokens=48, cin=512, cout=1000, bits=8, act="relu", want="xwbs"),
        # odd sizes, rows that start anywhere
        _case(_BACKWARD, "backward_odd", tokens=333, cin=1537, cout=1001, bits=8, act="silu", want="xwbs", pad=3),
        # frozen codes: scales and bias are learned, the input's gradient goes on to the layers before
        _case(_BACKWARD, "backward_frozen", tokens=2048, cin=4096, cout=4096, act="gelu", want="xbs"),
        # a step that trains the weights, which are quantized anew before each forward pass
        _case(_BACKWARD, "backward_train", tokens=4096, cin=4096, cout=4096, bits=8, act="gelu", want="xwb"),
        # the weight gradient alone, of many tokens (the first layer of a model)
        _case(_BACKWARD, "weight_gradient", tokens=8192, cin=4096, cout=4096, want="w"),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(("linear", "linear", "linear", "checkpoint", "backward", "backward"))
    if op == "checkpoint":
        return _case(_CHECKPOINT, tokens=log(1, 8192), cin=log(32, 11008), pad=rng.choice((0, 0, 1, 8)))
    cin, cout = log(64, 11008), log(64, 11008)
    if rng.random() < 0.5:   # most layers' widths are multiples of a vector
        cin, cout = cin + 63 & ~63, cout + 63 & ~63
    few = rng.random() < 0.4
    tokens = rng.randint(1, 32) if few else log(33, 4096)
    tokens = max(1, min(tokens, int(1.8e11 / (cin * cout))))
    kw = {"tokens": tokens, "cin": cin, "cout": cout, "bits": rng.choice((4, 8)),
          "act": rng.choice(("none", "relu", "gelu", "silu")), "pad": rng.choice((0, 0, 0, 1, 8))}
    if op == "linear":
        return _case(_LINEAR, dtype=rng.choice(("bf16", "fp16")), bias=rng.random() < 0.5, residual=rng.random() < 0.5,
                     save=rng.random() < 0.3, **kw)
    kw["tokens"] = max(1, min(tokens, int(0.9e11 / (cin * cout))))
    return _case(_BACKWARD, want=rng.choice(("x", "w", "xb", "xbs", "xwb", "xwbs")), **kw)


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _rows(v, pad):
    """`v` as a view of a buffer whose rows are `pad` elements longer."""
    wide = torch.empty((v.shape[0], v.shape[1] + pad), dtype=v.dtype, device=v.device)
    wide[:, :v.shape[1]] = v
    return wide[:, :v.shape[1]]


def _activations(g, tokens, features):
    """Activations with a few features that are much larger than the others, as language models have them."""
    v = _normal(g, tokens, features)
    return v * (1.0 + 15.0 * (torch.rand(features, generator=g, device="cuda") < 0.005))


def _pack(codes):
    """Two codes a byte, the even one in the low nibble; rows of ceil(cin / 2) bytes."""
    if codes.shape[1] % 2:
        codes = torch.cat((codes, codes.new_zeros(codes.shape[0], 1)), 1)
    u = codes.view(torch.uint8)
    return (u[:, 0::2] & 15 | (u[:, 1::2] & 15) << 4).view(torch.int8).contiguous()


def _unpack(codes, cin):
    u = codes.view(torch.uint8)
    both = torch.stack((u & 15, u >> 4), 2).view(u.shape[0], -1)[:, :cin].to(torch.int32)
    return both - 16 * (both > 7)


def _encode(v):
    """8-bit checkpoint of fp32 values: codes [rows, features rounded up to 32], exponents [rows, groups]."""
    rows, n = v.shape
    groups = -(-n // _GROUP)
    w = torch.zeros((rows, groups * _GROUP), dtype=torch.float32, device=v.device)
    w[:, :n] = v
    w = w.view(rows, groups, _GROUP)
    a = w.abs().amax(2)
    field = a.view(torch.int32) >> 23
    exps = torch.where(field == 255, 255, torch.clamp(field - 6, min=1))
    scale = torch.where(field == 255, 0, (254 - exps) << 23).view(torch.float32)   # 2^(127 - E)
    codes = torch.clamp(torch.round(torch.where(field[..., None] == 255, 0.0, w) * scale[..., None]), -127, 127)
    return codes.to(torch.int8).view(rows, groups * _GROUP), exps.to(torch.uint8)


def _decode(codes, exps, n):
    scale = (exps.to(torch.int32) << 23).view(torch.float32)   # 2^(E - 127), infinite for 255: 0 * inf is NaN
    rows = codes.shape[0]
    return (codes.view(rows, -1, _GROUP).to(torch.float32) * scale[..., None]).view(rows, -1)[:, :n]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    t, n = case["tokens"], case["cin"]
    state = dict(case)
    x = _activations(g, t, n)
    if case["op"] == "checkpoint":
        state["x"] = _rows(x.to(torch.bfloat16), case["pad"])
        return state
    m = case["cout"]
    w = _normal(g, m, n) * math.sqrt(1.0 / n) * torch.exp(0.3 * _normal(g, m, 1))
    qmax = 127 if case["bits"] == 8 else 7
    state["scales"] = w.abs().amax(1) / qmax
    codes = torch.clamp(torch.round(w / state["scales"][:, None]), -qmax, qmax).to(torch.int8)
    state["codes"] = _pack(codes) if case["bits"] == 4 else codes
    state["b"] = 0.1 * _normal(g, m)
    if case["op"] == "linear":
        dt = _TYPES[case["dtype"]]
        state["x"] = _rows(x.to(dt), case["pad"])
        state["bias_in"] = state["b"] if case["bias"] else None
        state["residual_in"] = _rows(_normal(g, t, m).to(dt), case["pad"]) if case["residual"] else None
        return state
    state["dy"] = _rows((1e-2 * _normal(g, t, m)).to(torch.bfloat16), case["pad"])
    state["x8"] = _encode(x.to(torch.bfloat16).float()) if "w" in case["want"] else None
    need_z = case["act"] != "none" or "s" in case["want"]
    state["z8"] = _encode(_normal(g, t, m) + state["b"]) if need_z else None
    return state


def _act(z, act):
    if act == "relu":
        return torch.where(z < 0, 0.0, z)
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * math.sqrt(0.5 / math.pi)
    if act == "silu":
        p = 1.0 / (1.0 + torch.exp(-z))
        return p * (1.0 + z * (1.0 - p))
    return torch.ones_like(z)


def _run_own(s):
    import paper_2202_07471_b200 as sq

    packed = s.get("bits") == 4
    if s["op"] == "checkpoint":
        return {"x": sq.squant_checkpoint_restore(sq.squant_checkpoint(s["x"]))}
    if s["op"] == "linear":
        y = sq.squant_linear(s["x"], s["codes"], s["scales"], s["bias_in"], residual=s["residual_in"], act=s["act"],
                             pack_int4=packed, checkpoint=s["save"])
        return {"y": y[0], "z": sq.squant_checkpoint_restore(y[1])} if s["save"] else {"y": y}
    x8 = sq.Checkpoint(*s["x8"], s["cin"]) if s["x8"] else None
    z8 = sq.Checkpoint(*s["z8"], s["cout"]) if s["z8"] else None
    want = s["want"]
    g = sq.squant_linear_backward(s["dy"], s["codes"], s["scales"], s["b"], cin=s["cin"], act=s["act"], pack_int4=packed, z=z8, x=x8,
                                  dx="x" in want, dweight="w" in want, dbias="b" in want, dscales="s" in want)
    return {"dx": g.dx, "dweight": g.dweight, "dbias": g.dbias, "dscales": g.dscales}


def run(s):
    if own:
        return _run_own(s)
    n = s["cin"]
    if s["op"] == "checkpoint":
        return {"x": _decode(*_encode(s["x"].float()), n).to(torch.bfloat16)}
    codes = (_unpack(s["codes"], n) if s["bits"] == 4 else s["codes"]).float()
    if s["op"] == "linear":
        z = (s["x"].float() @ codes.t()) * s["scales"]
        if s["bias_in"] is not None:
            z = z + s["bias_in"]
        y = _act(z, s["act"])
        if s["residual_in"] is not None:
            y = y + s["residual_in"].float()
        y = y.to(_TYPES[s["dtype"]])
        return {"y": y, "z": _decode(*_encode(z), s["cout"]).to(torch.bfloat16)} if s["save"] else {"y": y}
    want = s["want"]
    dz = s["dy"].float()
    z = _decode(*s["z8"], s["cout"]) if s["z8"] else None
    if s["act"] != "none":
        dz = dz * _act_slope(z, s["act"])
    return {"dx": ((dz * s["scales"]) @ codes).to(torch.bfloat16) if "x" in want else None,
            "dweight": (dz.t() @ _decode(*s["x8"], n)).to(torch.bfloat16) if "w" in want else None,
            "dbias": dz.sum(0) if "b" in want else None,
            "dscales": (dz * (z - s["b"])).sum(0) / s["scales"] if "s" in want else None}


def exact(case, seed):
    """The operators' definition in 64 bits, written apart from the forms above."""
    s = prepare(case, seed)
    n = case["cin"]
    f64 = torch.float64

    def eight(v):   # to the checkpoint's grid: 2^(floor(log2 of the group's largest) - 6), at least 2^-126
        rows, width = v.shape
        full = torch.nn.functional.pad(v, (0, -width % 32)).reshape(rows, -1, 32)
        top = torch.frexp(full.abs().amax(-1, keepdim=True)).exponent - 1
        step = torch.ldexp(torch.ones((), dtype=f64, device=v.device), torch.clamp(top - 6, min=-126))
        return (torch.clamp(torch.round(full / step), -127, 127) * step).reshape(rows, -1)[:, :width]

    def values(ck, width):
        q, e = ck
        step = torch.ldexp(torch.ones((), dtype=f64, device=q.device), e.to(torch.int32) - 127)
        return (q.to(f64) * step.repeat_interleave(32, dim=1))[:, :width]

    if case["op"] == "checkpoint":
        return {"x": eight(s["x"].to(f64))}
    if case["bits"] == 4:
        raw = s["codes"].to(torch.int64)
        low, high = (raw + 8) % 16 - 8, torch.div(raw, 16, rounding_mode="floor")
        codes = torch.empty((raw.shape[0], 2 * raw.shape[1]), dtype=f64, device=raw.device)
        codes[:, 0::2], codes[:, 1::2] = low.to(f64), high.to(f64)
        codes = codes[:, :n]
    else:
        codes = s["codes"].to(f64)
    weights = codes * s["scales"].to(f64)[:, None]

    def phi(v):   # the normal distribution function
        return 0.5 * torch.special.erfc(-v / math.sqrt(2.0))

    if case["op"] == "linear":
        z = torch.mm(s["x"].to(f64), weights.T)
        if case["bias"]:
            z += s["bias_in"].to(f64)
        y = {"none": lambda: z, "relu": lambda: z.clamp(min=0), "gelu": lambda: z * phi(z), "silu": lambda: z * torch.sigmoid(z)}[case["act"]]()
        if case["residual"]:
            y = y + s["residual_in"].to(f64)
        return {"y": y, "z": eight(z)} if case["save"] else {"y": y}
    dz = s["dy"].to(f64)
    z = values(s["z8"], case["cout"]) if s["z8"] else None
    if case["act"] == "relu":
        dz = torch.where(z > 0, dz, torch.zeros_like(dz))
    elif case["act"] == "gelu":
        dz = dz * (phi(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi))
    elif case["act"] == "silu":
        p = torch.sigmoid(z)
        dz = dz * (p + z * p * (1 - p))
    out = {"dx": None, "dweight": None, "dbias": None, "dscales": None}
    if "x" in case["want"]:
        out["dx"] = dz @ weights
    if "w" in case["want"]:
        out["dweight"] = dz.T @ values(s["x8"], n)
    if "b" in case["want"]:
        out["dbias"] = dz.sum(dim=0)
    if "s" in case["want"]:
        out["dscales"] = (dz * (z - s["b"].to(f64)) / s["scales"].to(f64)).sum(dim=0)
    return out


def work(case):
    t, n = case["tokens"], case["cin"]
    eighth = 1.0 + 1.0 / _GROUP   # bytes of a checkpoint's element
    if case["op"] == "checkpoint":
        return {"bytes": t * n * (2 + eighth) * 2, "flops": 0}
    m = case["cout"]
    codes = m * n * case["bits"] // 8 + 4 * m
    if case["op"] == "linear":
        moved = 2 * t * n + codes + 2 * t * m * (2 if case["residual"] else 1) + 4 * m * case["bias"]
        return {"bytes": moved + (t * m * (2 * eighth + 2) if case["save"] else 0), "flops": 2.0 * t * m * n}
    want = case["want"]
    moved = 2 * t * m + (t * m * eighth if case["act"] != "none" or "s" in want else 0)
    moved += codes + 2 * t * n if "x" in want else 0
    moved += t * n * eighth + 2 * m * n if "w" in want else 0
    moved += 4 * m * (("b" in want) + ("s" in want))
    return {"bytes": moved, "flops": 2.0 * t * m * n * (("x" in want) + ("w" in want))}
