"""A small, self-terminating case of the large-layer workload for profilers.

  python -m paper_2202_07471_b200.profile_case [--channels M] [--launches L] [--mode 7]
  python -m paper_2202_07471_b200.profile_case --workload resnet50 [--launches L]
  python -m paper_2202_07471_b200.profile_case --layer 128x65541x1x1 [--pack] [--no-sums] [--bits B]
  python -m paper_2202_07471_b200.profile_case --linear 2048x4096x11008 [--pack] [--backward]

Quantizes one [M, 2048, 3, 3] layer (default M = 4096: 302 MB of weights, larger than L2, a few
hundred MB on the device) L times through the C ABI.  Values follow the large-layer recipe
(seeded normal weights with a per-channel log-uniform scale).  With --workload NAME the whole
model of that name (resnet18, resnet50, mobilenetv2, mixed_kernels) is quantized in one call instead,
with --layer one layer of that shape (normal weights; --pack: packed int4 codes).  With --linear
TOKENSxCINxCOUT a linear layer is quantized and called (--backward: its gradients with gelu, from 8-bit checkpoints).
"""
from __future__ import annotations

import argparse

import numpy as np
import torch

from . import binding as sq
from . import linear
from . import workloads as W


def main() -> None:
    ap = argparse.ArgumentParser()
    ap.add_argument("--channels", type=int, default=4096)
    ap.add_argument("--launches", type=int, default=3)
    ap.add_argument("--bits", type=int, default=4)
    ap.add_argument("--mode", type=int, default=sq.MODE_EKC)
    ap.add_argument("--workload", default="large_layer")
    ap.add_argument("--layer", default="", help="cout x cin x kh x kw")
    ap.add_argument("--pack", action="store_true")
    ap.add_argument("--no-sums", action="store_true", help="no kernel and channel error sums")
    ap.add_argument("--linear", default="", help="tokens x cin x cout")
    ap.add_argument("--backward", action="store_true")
    args = ap.parse_args()
    if args.linear:
        tokens, cin, cout = (int(v) for v in args.linear.split("x"))
        g = torch.Generator("cuda").manual_seed(0)
        buf = sq.alloc_outputs(torch.randn((cout, cin), device="cuda", generator=g) / cin ** 0.5, False, False, pack_int4=args.pack)
        sq.squant_quantize_model([buf], bits=4 if args.pack else 8, flags=sq.FLAG_NARROW_RANGE | (sq.FLAG_PACK_INT4 if args.pack else 0))
        x = torch.randn((tokens, cin), device="cuda", generator=g).bfloat16()
        dy = torch.randn((tokens, cout), device="cuda", generator=g).bfloat16()
        if args.backward:
            x8, z8 = linear.squant_checkpoint(x), linear.squant_checkpoint(dy)
        for _ in range(args.launches):
            if args.backward:
                linear.squant_linear_backward(dy, buf.codes, buf.scales, cin=cin, act="gelu", pack_int4=args.pack, z=z8, x=x8, dweight=True, dbias=True)
            else:
                linear.squant_linear(x, buf.codes, buf.scales, pack_int4=args.pack)
        sq.squant_device_status()
        print(f"ok: {args.launches} calls of a linear layer, {tokens} tokens, {cin} to {cout}")
        return
    if args.layer:
        shape = [int(v) for v in args.layer.split("x")]
        w = torch.randn(shape, device="cuda", generator=torch.Generator("cuda").manual_seed(0)) * (2.0 / (shape[1] * shape[2] * shape[3])) ** 0.5
        buf = sq.alloc_outputs(w, kernel_err=not args.no_sums, channel_err=not args.no_sums, pack_int4=args.pack)
        flags = sq.FLAG_NARROW_RANGE | (sq.FLAG_PACK_INT4 if args.pack else 0)
        call = sq.ModelCall([buf], bits=args.bits, mode=args.mode, flags=flags)
        for _ in range(args.launches):
            call.run()
        sq.squant_device_status()
        print(f"ok: {args.launches} launches of {shape}, {w.numel()} weights each, {sq.squant_plan_kernels([buf], args.bits, args.mode, flags)[0]} kernel")
        return
    if args.workload != "large_layer":
        wl = W.WORKLOADS[args.workload]
        ws = [torch.from_numpy(W.layer_weights(wl, i, seed=0, threads=8)).cuda() for i in range(len(wl.shapes))]
        call = sq.ModelCall([sq.alloc_outputs(w) for w in ws], bits=args.bits, mode=args.mode)
        for _ in range(args.launches):
            call.run()
        sq.squant_device_status()
        print(f"ok: {args.launches} launches of {args.workload}, {sum(w.numel() for w in ws)} weights each")
        return
    wl = W.WORKLOADS["large_layer"]
    m = min(args.channels, 2048)
    reps = (args.channels + m - 1) // m
    parts = [W.layer_weights(wl, i % len(wl.shapes), seed=0, channels=slice(0, m), threads=8) for i in range(reps)]
    w = torch.from_numpy(np.concatenate(parts)[:args.channels]).cuda()
    bufs = sq.alloc_outputs(w)
    call = sq.ModelCall([bufs], bits=args.bits, mode=args.mode)
    for _ in range(args.launches):
        call.run()
    sq.squant_device_status()
    print(f"ok: {args.launches} launches of [{args.channels}, 2048, 3, 3], {w.numel()} weights each")


if __name__ == "__main__":
    main()
