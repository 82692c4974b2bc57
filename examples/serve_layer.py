"""A quantized decoder layer as it is served: learn a transform, quantize and pack the projections that share it, and run
tokens through the norm (residual added, inverse transform, 8 bits) and the packed products.

    python examples/serve_layer.py [--d 4608] [--outs 4096,2048,36864] [--tokens 1] [--k 128] [--group 128] [--bits 4]

The weights are random stand-ins of the 27B-shaped layer's q, k and gate projections, which read the same normalised
residual stream and so share one transform along their inputs.  Prints, per projection, how far the served result is from the
unquantized layer's, and what a step takes."""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2511_19705_amd import cafeq  # noqa: E402

DEVICE = "cuda:0"


def rotations(nb, k, gen):
    """Haar rotations, the initial transform."""
    q, r = torch.linalg.qr(torch.randn((nb, k, k), generator=gen, device=DEVICE, dtype=torch.float64))
    return (q * torch.sign(torch.diagonal(r, dim1=1, dim2=2))[:, None, :]).float().contiguous()


def quantize(weights, k, bits, group, steps, gen):
    """(packed projections, inverse blocks): the transform learned on the largest of them, codes and scales of all at it."""
    largest = max(weights, key=lambda w: w.shape[0])
    T = rotations(largest.shape[1] // k, k, gen)
    Tinv, _, status = cafeq.optimize_single(largest, T, bits, group, lr=0.5, steps=steps)
    assert not status.any(), "a block of the transform is singular"
    packed = []
    for w in weights:
        _, _, codes, scales = cafeq.proxy_loss_fwd_bwd(w, T, Tinv, bits, group, want_grad=False, want_codes=True)
        packed.append(cafeq.pack_nibbles(codes, scales, group))
    return packed, Tinv


def step(x, residual, gain, Tinv, packed, group):
    """One layer's entry: (sum, projections).  x: what the layer before added to the residual stream."""
    a = cafeq.norm_quantize(x, gain, residual=residual, gain_offset=1.0, Tinv=Tinv, group=group)
    return a.sum, [cafeq.infer_packed(a.codes, w, xscales=a.scales, xgroup=group, dtype=torch.bfloat16) for w in packed]


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--d", type=int, default=4608)
    ap.add_argument("--outs", default="4096,2048,36864")
    ap.add_argument("--tokens", type=int, default=1)
    ap.add_argument("--k", type=int, default=128)
    ap.add_argument("--group", type=int, default=128)
    ap.add_argument("--bits", type=int, default=4, choices=(2, 3, 4))
    ap.add_argument("--steps", type=int, default=10)
    a = ap.parse_args(argv)
    gen = torch.Generator(device=DEVICE).manual_seed(0)
    weights = [torch.randn((int(o), a.d), generator=gen, device=DEVICE) * 0.02 for o in a.outs.split(",")]
    packed, Tinv = quantize(weights, a.k, a.bits, a.group, a.steps, gen)
    gain = torch.randn(a.d, generator=gen, device=DEVICE) * 0.2
    x = torch.randn((a.tokens, a.d), generator=gen, device=DEVICE).bfloat16()
    residual = torch.randn((a.tokens, a.d), generator=gen, device=DEVICE).bfloat16()
    total, ys = step(x, residual, gain, Tinv, packed, a.group)
    h = x.double() + residual.double()
    y = h / (h.square().mean(1, keepdim=True) + 1e-6).sqrt() * (1.0 + gain.double())
    errors = []
    for w, got in zip(weights, ys):
        want = y @ w.double().t()
        errors.append(float((got.double() - want).norm() / want.norm()))
        print("%6d x %d, %d bits: relative error %.4f" % (w.shape[0], w.shape[1], a.bits, errors[-1]))
    for _ in range(20):
        step(x, residual, gain, Tinv, packed, a.group)
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(100):
        step(x, residual, gain, Tinv, packed, a.group)
    torch.cuda.synchronize()
    t = (time.perf_counter() - t) / 100
    nbytes = sum(w.data.numel() for w in packed) + 4 * Tinv.numel()
    print("%d token(s): %.1f us a step, %.0f GB/s of weights" % (a.tokens, t * 1e6, nbytes / t / 1e9))
    return errors


if __name__ == "__main__":
    main()
