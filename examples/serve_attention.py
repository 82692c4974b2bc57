"""A quantized attention layer as it is served: prompts, continuations that share them, and single tokens in a captured graph.

    python examples/serve_attention.py [--d 4608] [--heads_q 32] [--heads 16] [--head 128] [--prompts 512,300] [--forks 2] [--steps 32]

The weights are random stand-ins of the 27B-shaped layer's q, k, v and o, quantized to 4 bits with groups and packed; keys and values are held in 8
bits with a scale for each block of tokens and head.  A step: norm with 8 bits, one packed product for q, k and v, norm and position of each head, room in
the pages, keys and values into them, attention, 8 bits, the packed output product.  Prints how far the last prompt's result is from the layer with the same
weights in float64, and what a step of single tokens takes."""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2511_19705_amd import cafeq  # noqa: E402

DEVICE = "cuda:0"
GROUP = 128


def ints(values):
    return torch.tensor(list(values), dtype=torch.int32, device=DEVICE)


class Layer:
    """One attention layer and its cache."""

    def __init__(self, d, heads_q, heads, head, rows, tokens, gen, block=64, softcap=0.0, window=0):
        self.d, self.heads_q, self.heads, self.head, self.softcap, self.window = d, heads_q, heads, head, softcap, window
        self.dense = []
        packed = []
        for out, width in (((heads_q + 2 * heads) * head, d), (d, heads_q * head)):
            w = torch.randn((out, width), generator=gen, device=DEVICE) * width ** -0.5
            codes, scales, _ = cafeq.rtn_quantize(w, 4, GROUP)
            packed.append(cafeq.pack_nibbles(codes, scales, GROUP))
            self.dense.append(codes.double() * scales.double().repeat_interleave(GROUP, 1))
        self.qkv, self.o = packed
        self.gain, self.gain_q, self.gain_k = (torch.randn(n, generator=gen, device=DEVICE) * 0.2 for n in (d, head, head))
        self.freq, self.amplitude = cafeq.rotary_frequencies(head, device=DEVICE)
        width = -(-tokens // block)
        self.cache = cafeq.kv_cache(rows, rows * width, heads, head, block=block, width=width, device=DEVICE)

    def step(self, x, starts, longest):
        """New tokens x [n][d] of the rows that starts gives; their result [n][d].  Without room for them (cache.missing, on the device) the cache stays as it is."""
        n, (hq, h, hd) = x.shape[0], (self.heads_q, self.heads, self.head)
        a = cafeq.norm_quantize(x, self.gain, gain_offset=1.0, group=GROUP)
        y = cafeq.infer_packed(a.codes, self.qkv, xscales=a.scales, xgroup=GROUP, dtype=torch.bfloat16)
        q, k, v = (y[:, at * hd:(at + m) * hd].unflatten(1, (m, hd)) for at, m in ((0, hq), (hq, h), (hq + h, h)))
        positions = cafeq.cache_reserve(self.cache, starts, n).positions
        cafeq.rotate_heads(q, k, positions, self.freq, norm=True, gain_q=self.gain_q, gain_k=self.gain_k, gain_offset=1.0, amplitude=self.amplitude,
                           out_q=q, out_k=k)
        cafeq.cache_append(self.cache, k, v, starts, longest=longest)
        z = cafeq.cache_attend(self.cache, q, starts, longest=longest, softcap=self.softcap, window=self.window)
        b = cafeq.norm_quantize(z.flatten(1), norm=False, group=GROUP)
        return cafeq.infer_packed(b.codes, self.o, xscales=b.scales, xgroup=GROUP, dtype=torch.bfloat16)

    def exact(self, x):
        """The result for one prompt x in float64: the same weights, nothing else rounded."""
        n, (hq, h, hd) = x.shape[0], (self.heads_q, self.heads, self.head)
        x = x.double()
        y = (x / (x.square().mean(1, keepdim=True) + 1e-6).sqrt() * (1.0 + self.gain.double())) @ self.dense[0].t()
        q, k, v = (y[:, at * hd:(at + m) * hd].reshape(n, m, hd) for at, m in ((0, hq), (hq, h), (hq + h, h)))
        angle = torch.arange(n, device=DEVICE, dtype=torch.float64)[:, None] * self.freq
        c, s = angle.cos()[:, None], angle.sin()[:, None]

        def turn(t, gain):
            t = t / (t.square().mean(2, keepdim=True) + 1e-6).sqrt() * (1.0 + gain.double())
            a, b = t[:, :, :hd // 2], t[:, :, hd // 2:]
            return torch.cat((a * c - b * s, a * s + b * c), 2)

        q, k = turn(q, self.gain_q), turn(k, self.gain_k)
        at = torch.arange(n, device=DEVICE)
        out = torch.empty_like(q)
        for j in range(hq):
            p = q[:, j] @ k[:, j * h // hq].t() * hd ** -0.5
            if self.softcap:
                p = self.softcap * torch.tanh(p / self.softcap)
            p[at[None, :] > at[:, None]] = float("-inf")
            if self.window:
                p[at[None, :] <= at[:, None] - self.window] = float("-inf")
            out[:, j] = torch.softmax(p, 1) @ v[:, j * h // hq]
        return out.flatten(1) @ self.dense[1].t()


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--d", type=int, default=4608)
    ap.add_argument("--heads_q", type=int, default=32)
    ap.add_argument("--heads", type=int, default=16)
    ap.add_argument("--head", type=int, default=128)
    ap.add_argument("--prompts", default="512,300")
    ap.add_argument("--forks", type=int, default=2, help="continuations of each prompt")
    ap.add_argument("--steps", type=int, default=32)
    ap.add_argument("--softcap", type=float, default=0.0)
    a = ap.parse_args(argv)
    gen = torch.Generator(device=DEVICE).manual_seed(0)
    prompts = [int(p) for p in a.prompts.split(",")]
    rows = len(prompts) * a.forks
    layer = Layer(a.d, a.heads_q, a.heads, a.head, rows, max(prompts) + a.steps + 8, gen, softcap=a.softcap)
    starts = [0]
    for i in range(rows):
        starts.append(starts[-1] + (prompts[i] if i < len(prompts) else 0))
    x = torch.randn((starts[-1], a.d), generator=gen, device=DEVICE).bfloat16()
    y = layer.step(x, ints(starts), max(prompts))
    last = slice(starts[len(prompts) - 1], starts[len(prompts)])
    want = layer.exact(x[last])
    error = float((y[last].double() - want).norm() / want.norm())
    print("prompts of %s tokens: relative error %.4f" % (a.prompts, error))
    # each prompt goes on in `forks` rows, which share its pages until they write to them
    cafeq.cache_reorder(layer.cache, ints(i % len(prompts) for i in range(rows)))
    one, token = ints(range(rows + 1)), torch.randn((rows, a.d), generator=gen, device=DEVICE).bfloat16()
    for _ in range(2):
        layer.step(token, one, 1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.step(token, one, 1)
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(a.steps):
        graph.replay()
    torch.cuda.synchronize()
    t = (time.perf_counter() - t) / a.steps
    lengths = layer.cache.lengths.tolist()
    used = int(cafeq.cache_compact(layer.cache))
    print("%d rows of %d to %d tokens on %d pages: %.1f us a step" % (rows, min(lengths), max(lengths), used, t * 1e6))
    return error, lengths, used


if __name__ == "__main__":
    main()
