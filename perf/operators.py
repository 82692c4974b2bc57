"""The serving side of a quantized decoder layer as timed cases: activations made ready in 8 bits, and products with
packed 4-bit weights.

Two operators and both together:
  norm    h = x + residual; y = h / sqrt(mean h^2 + eps) * (1 + gain); z = y through blocks of an inverse transform
          (optional); then 8 bits with a scale per group of columns, or z as it is
  linear  Y[t][o] = sum_c scale[o][c / g] code[o][c] X[t][c], codes of 4 bits, activations in float32, bfloat16 or
          8 bits with scales, from one token to a long prompt
  layer   the norm and the projections that read its codes

A case is a dict of plain values:
  kind            norm | linear | layer
  tokens          rows of activations
  d               norm, layer: columns
  k               norm, layer: block size of the transform, 0 = none
  residual        norm: whether a residual is added (and the sum written)
  dtype           storage of the activations: f32 | bf16 | i8 (linear only; bf16 for what such a product returns)
  group           norm: columns a scale of the 8-bit output, 0 = the whole row, -1 = no codes, the values in `dtype`
  rows, cols      linear: the weight [rows][cols]
  wgroup, xgroup  linear, layer: columns a scale of the weights, of 8-bit activations (0 = the whole row)
  outs            layer: rows of the projections, as text "4096,2048"
Sizes are those of the 2B-, 9B- and 27B-shaped layers of ``workloads`` and between them, with rows that fill no tile.
"""
from __future__ import annotations

import math

import torch

own = False
DEVICE = "cuda:0"
EPS = 1e-6
_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ----------------------------------------------------------------------------------------------------
# the cases
# ----------------------------------------------------------------------------------------------------
def _norm(tokens, d, dtype, residual, k, group):
    return dict(kind="norm", tokens=tokens, d=d, dtype=dtype, residual=residual, k=k, group=group)


def _linear(tokens, rows, cols, dtype, wgroup, xgroup=0):
    return dict(kind="linear", tokens=tokens, rows=rows, cols=cols, dtype=dtype, wgroup=wgroup, xgroup=xgroup)


def _layer(tokens, d, k, outs, wgroup):
    return dict(kind="layer", tokens=tokens, d=d, k=k, outs=outs, wgroup=wgroup, xgroup=wgroup)


def listed():
    return [
        # One decoded token of the 2B-shaped model before a projection without a transform: the smallest call.
        dict(name="norm_1_2b", **_norm(1, 2304, "bf16", True, 0, 128)),
        # One decoded token of the 9B-shaped model before a projection whose transform has blocks of 128.
        dict(name="norm_1_9b_k128", **_norm(1, 3584, "bf16", True, 128, 128)),
        # A prompt of the 9B-shaped model, one scale a token.
        dict(name="norm_4096_9b_rows", **_norm(4096, 3584, "bf16", True, 0, 0)),
        # A prompt of the 27B-shaped model through blocks of 128.
        dict(name="norm_2048_27b_k128", **_norm(2048, 4608, "bf16", True, 128, 128)),
        # A batch that fills no tile, in float32, through blocks of 64, for a consumer that reads no codes.
        dict(name="norm_333_ragged_f32", **_norm(333, 2880, "f32", False, 64, -1)),
        # One decoded token through the 2B-shaped down projection (the matrix of the block-size table).
        dict(name="linear_1_2b_down", **_linear(1, 2304, 9216, "i8", 128, 128)),
        # One decoded token through the 27B-shaped gate projection, activations in bfloat16.
        dict(name="linear_1_27b_gate_bf16", **_linear(1, 36864, 4608, "bf16", 128)),
        # Sixteen sequences decoded together through the 9B-shaped down projection.
        dict(name="linear_16_9b_down", **_linear(16, 3584, 14336, "i8", 128, 128)),
        # A ragged batch through a matrix whose rows fill no tile, groups of 32, float32 activations.
        dict(name="linear_37_ragged_f32", **_linear(37, 1147, 2880, "f32", 32)),
        # A short prompt through the 9B-shaped up projection, activations in bfloat16.
        dict(name="linear_512_9b_up_bf16", **_linear(512, 14336, 3584, "bf16", 128)),
        # A long prompt through the 27B-shaped down projection, one activation scale a token: the largest call.
        dict(name="linear_4096_27b_down", **_linear(4096, 4608, 36864, "i8", 128, 0)),
        # Eight sequences: the norm of a 27B-shaped layer, its transform, and the q, k and gate projections that share it.
        dict(name="layer_8_27b_q_k_gate", **_layer(8, 4608, 128, "4096,2048,36864", 128)),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def _axis(rng, lo, hi, unit):
    v = max(unit, _log_int(rng, lo, hi) // unit * unit)
    return v + unit if v == 3072 else v


def draw(rng):
    kind = rng.choice(("norm", "norm", "linear", "linear", "linear", "layer"))
    if kind == "norm":
        k = rng.choice((0, 0, 32, 64, 128, 256))
        group = rng.choice((-1, 0, 32, 64, 128, 128, 256))
        d = _axis(rng, 256, 14336, max(k, group, 32))
        tokens = _log_int(rng, 1, min(4096, max(1, 14_000_000 // d)))
        return _norm(tokens, d, rng.choice(("f32", "bf16", "bf16")), rng.random() < 0.7, k, group)
    wgroup = rng.choice((32, 64, 128, 128, 128, 256, 0))
    if kind == "layer":
        k = rng.choice((32, 64, 128, 256))
        d = _axis(rng, 512, 4608, max(k, wgroup, 32))
        outs = ",".join(str(_log_int(rng, 64, 9216)) for _ in range(rng.choice((1, 2, 3))))
        return _layer(_log_int(rng, 1, 512), d, k, outs, wgroup)
    dtype = rng.choice(("i8", "i8", "bf16", "f32"))
    cols = _axis(rng, 256, 36864, max(wgroup, 32))
    rows = _log_int(rng, 64, min(36864, 170_000_000 // cols))
    tokens = _log_int(rng, 1, 4096)
    return _linear(tokens, rows, cols, dtype, wgroup, rng.choice((wgroup, 0)) if dtype == "i8" else 0)


# ----------------------------------------------------------------------------------------------------
# inputs
# ----------------------------------------------------------------------------------------------------
def _spread(v, group, n, width):
    """One value a group along the rows of a matrix of `width` columns."""
    return v.reshape(n, -1, 1).expand(n, v.numel() // max(n, 1), group or width).reshape(n, width)


def _round_to_grid(w, group, top):
    """Codes on the symmetric grid of `top` and a scale a group (0: the row)."""
    n, width = w.shape
    v = w.reshape(n, -1, group or width)
    a = v.abs().amax(2, keepdim=True)
    codes = torch.round(v * (top / a)).to(torch.int8).reshape(n, width)
    return codes, (a / top).reshape(n, -1).contiguous()


def _weight(rows, cols, group, gen):
    """Codes and scales of heavy-tailed weights of a standard deviation of 0.02, on the grid of 4 bits."""
    w = torch.randn((rows, cols), generator=gen, device=DEVICE)
    w.mul_(torch.rand((rows, cols), generator=gen, device=DEVICE).clamp_(min=1e-3).pow_(-1.0 / 4).mul_(0.014))
    return _round_to_grid(w, group, 7.0)


def _stream(tokens, d, gen):
    """A residual stream: unit Gaussians, a few channels thirty times larger in every token."""
    x = torch.randn((tokens, d), generator=gen, device=DEVICE)
    x[:, torch.randperm(d, generator=gen, device=DEVICE)[:max(1, d // 512)]] *= 30.0
    return x


def _inverses(d, k, gen):
    """Blocks near rotations, as the inverses of learned transforms are."""
    q, r = torch.linalg.qr(torch.randn((d // k, k, k), generator=gen, device=DEVICE))
    q = q * torch.sign(torch.diagonal(r, dim1=1, dim2=2))[:, None, :]
    return (q + torch.randn(q.shape, generator=gen, device=DEVICE) * (0.05 / math.sqrt(k))).contiguous()


def _inputs(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(int(seed))
    c, s = case, {"case": dict(case)}
    if c["kind"] == "linear":
        s["codes"], s["scales"] = _weight(c["rows"], c["cols"], c["wgroup"], gen)
        x = _stream(c["tokens"], c["cols"], gen)
        if c["dtype"] == "i8":
            s["x"], s["xscales"] = _round_to_grid(x, c["xgroup"], 127.0)
        else:
            s["x"], s["xscales"] = x.to(_TYPES[c["dtype"]]), None
        return s
    dtype = _TYPES[c.get("dtype", "bf16")]
    s["x"] = (_stream(c["tokens"], c["d"], gen) * 0.3).to(dtype)
    s["residual"] = _stream(c["tokens"], c["d"], gen).to(dtype) if c.get("residual", True) else None
    s["gain"] = torch.randn(c["d"], generator=gen, device=DEVICE) * 0.2
    s["P"] = _inverses(c["d"], c["k"], gen) if c["k"] else None
    if c["kind"] == "layer":
        s["weights"] = [_weight(int(o), c["d"], c["wgroup"], gen) for o in c["outs"].split(",")]
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        # a serving program keeps its weights packed, not as one byte a code
        from paper_2511_19705_amd import cafeq
        g = case.get("wgroup")
        if case["kind"] == "linear":
            s["packed"] = cafeq.pack_nibbles(s.pop("codes"), s.pop("scales"), g)
        elif case["kind"] == "layer":
            s["packed"] = [cafeq.pack_nibbles(q, v, g) for q, v in s.pop("weights")]
    return s


# ----------------------------------------------------------------------------------------------------
# one pass: the plain forms, and the framework's
# ----------------------------------------------------------------------------------------------------
def _plain_norm(s, group):
    """(sum, z in float32 or the values of its codes, scales)."""
    x, P = s["x"], s["P"]
    n, d = x.shape
    h = x.float() if s["residual"] is None else x.float() + s["residual"].float()
    z = h * torch.rsqrt(h.square().mean(1, keepdim=True) + EPS) * (1.0 + s["gain"])
    if P is not None:
        nb, k, _ = P.shape
        blocks = z.reshape(n, nb, k).transpose(0, 1).contiguous()
        z = torch.bmm(blocks, P.transpose(1, 2).contiguous()).transpose(0, 1).reshape(n, d)
    if group < 0:
        return h, z, None
    v = z.reshape(n, -1, group or d)
    a = v.abs().amax(2, keepdim=True)
    scales = a / 127.0
    inv = torch.where(a > 0, 127.0 / a, torch.zeros_like(a))
    return h, (torch.round(v * inv) * scales).reshape(n, d), scales.reshape(n, -1)


def _plain_linear(x, codes, scales, group):
    rows, cols = codes.shape
    return x @ (codes.float() * _spread(scales, group, rows, cols)).t()


def _run_plain(s):
    c = s["case"]
    if c["kind"] == "linear":
        x = s["x"].float()
        if s["xscales"] is not None:
            x = x * _spread(s["xscales"], c["xgroup"], *x.shape)
        y = _plain_linear(x, s["codes"], s["scales"], c["wgroup"])
        return {"y": y.to(torch.float32 if c["dtype"] == "f32" else torch.bfloat16)}
    if c["kind"] == "norm":
        h, z, scales = _plain_norm(s, c["group"])
        kept = h.to(s["x"].dtype) if c["residual"] else None
        if c["group"] < 0:
            return {"sum": kept, "values": z.to(s["x"].dtype)}
        return {"sum": kept, "values": z.to(torch.bfloat16), "scales": scales}
    h, z, _ = _plain_norm(s, c["xgroup"])
    return {"sum": h.to(s["x"].dtype), "y": [_plain_linear(z, q, v, c["wgroup"]).to(torch.bfloat16) for q, v in s["weights"]]}


def _run_own(s):
    from paper_2511_19705_amd import cafeq
    c = s["case"]
    if c["kind"] == "linear":
        out = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
        return {"y": cafeq.infer_packed(s["x"], s["packed"], xscales=s["xscales"], xgroup=c["xgroup"], dtype=out)}
    if c["kind"] == "norm":
        group = c["group"]
        # `values`: what the codes stand for, or the result itself where no codes are asked for
        r = cafeq.norm_quantize(s["x"], s["gain"], residual=s["residual"], eps=EPS, gain_offset=1.0, Tinv=s["P"],
                                group=None if group < 0 else group, values=s["x"].dtype if group < 0 else torch.bfloat16)
        return {"sum": r.sum, "values": r.values, "scales": r.scales} if group >= 0 else {"sum": r.sum, "values": r.values}
    r = cafeq.norm_quantize(s["x"], s["gain"], residual=s["residual"], eps=EPS, gain_offset=1.0, Tinv=s["P"], group=c["xgroup"])
    return {"sum": r.sum, "y": [cafeq.infer_packed(r.codes, w, xscales=r.scales, xgroup=c["xgroup"], dtype=torch.bfloat16)
                                for w in s["packed"]]}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ----------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ----------------------------------------------------------------------------------------------------
def _exact_norm(s, group):
    h = s["x"].double()
    if s["residual"] is not None:
        h = h + s["residual"].double()
    y = h / torch.sqrt((h * h).sum(1, keepdim=True) / h.shape[1] + EPS) * (1.0 + s["gain"].double())
    z = y
    if s["P"] is not None:
        k = s["P"].shape[1]
        z = torch.cat([y[:, b * k:(b + 1) * k] @ s["P"][b].double().t().contiguous() for b in range(s["P"].shape[0])], 1)
    if group < 0:
        return h, z, None
    parts = z.split(group or z.shape[1], 1)
    scales = torch.stack([p.abs().amax(1) for p in parts], 1) / 127.0
    values = torch.cat([torch.where(a[:, None] > 0, torch.round(p / a[:, None]) * a[:, None], torch.zeros_like(p))
                        for p, a in zip(parts, scales.unbind(1))], 1)
    return h, values, scales


def _exact_product(x, codes, scales, group):
    """A product over each scale group, times its scales, added up."""
    g = group or codes.shape[1]
    if codes.shape[1] // g > 64:      # short groups: the weights themselves
        w = codes.double().mul_(scales.double().repeat_interleave(g, 1))
        return x @ w.t()
    y = torch.zeros((x.shape[0], codes.shape[0]), dtype=torch.float64, device=x.device)
    for i in range(codes.shape[1] // g):
        y += (x[:, i * g:(i + 1) * g].contiguous() @ codes[:, i * g:(i + 1) * g].double().t()) * scales[:, i].double()
    return y


def exact(case, seed):
    c, s = case, _inputs(case, seed)
    if c["kind"] == "linear":
        x = s["x"].double()
        if s["xscales"] is not None:
            x = x * s["xscales"].double().repeat_interleave(c["xgroup"] or c["cols"], 1)
        return {"y": _exact_product(x, s["codes"], s["scales"], c["wgroup"])}
    if c["kind"] == "norm":
        h, z, scales = _exact_norm(s, c["group"])
        kept = h if c["residual"] else None
        return {"sum": kept, "values": z} if c["group"] < 0 else {"sum": kept, "values": z, "scales": scales}
    h, z, _ = _exact_norm(s, c["xgroup"])
    return {"sum": h, "y": [_exact_product(z, q, v, c["wgroup"]) for q, v in s["weights"]]}


# ----------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ----------------------------------------------------------------------------------------------------
def _norm_work(c, values):
    n, d = c["tokens"], c["d"]
    size = 4 if c.get("dtype", "bf16") == "f32" else 2
    res = c.get("residual", True)
    group = c["xgroup"] if c["kind"] == "layer" else c["group"]
    size_out = size if group < 0 else (1 + (2 if values else 0))
    scales = 0 if group < 0 else 4 * n * (d // (group or d))
    return (n * d * (size * (3 if res else 1) + size_out) + scales + 4 * d + 4 * d * c["k"], 2.0 * n * d * c["k"] + 8.0 * n * d)


def _linear_work(n, rows, cols, wgroup, x_bytes, y_size):
    return (rows * cols // 2 + 4 * rows * (cols // (wgroup or cols)) + x_bytes + n * rows * y_size, 2.0 * n * rows * cols)


def work(case):
    c, n = case, case["tokens"]
    if c["kind"] == "norm":
        b, f = _norm_work(c, True)
    elif c["kind"] == "linear":
        x = n * c["cols"] * {"f32": 4, "bf16": 2, "i8": 1}[c["dtype"]]
        if c["dtype"] == "i8":
            x += 4 * n * (c["cols"] // (c["xgroup"] or c["cols"]))
        b, f = _linear_work(n, c["rows"], c["cols"], c["wgroup"], x, 4 if c["dtype"] == "f32" else 2)
    else:
        b, f = _norm_work(c, False)
        x = n * c["d"] + 4 * n * (c["d"] // (c["xgroup"] or c["d"]))
        for o in c["outs"].split(","):
            more = _linear_work(n, int(o), c["d"], c["wgroup"], x, 2)
            b, f = b + more[0], f + more[1]
    return {"bytes": float(b), "flops": float(f)}
