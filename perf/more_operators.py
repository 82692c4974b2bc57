"""What stands between the projections of a quantized decoder layer as timed cases: the norm and the positions of queries
and keys, a cache of keys and values in 8 bits, attention over it, and its pages.

Operators:
  rotate   queries and keys of every head: root-mean-square norm (optional), then pairs of channels turned by position x frequency
  append   new keys and values into the pages of their sequences: int8 codes with a scale for each block of tokens and head; a
           block that already holds tokens takes the larger scale, its codes go over to it
  attend   attention of new tokens over the cache, from one token a sequence to whole prompts
  fork     continuations of prompts: rows of the page table taken over from others, a place for one token more, shared blocks that
           are appended to copied first
  compact  one batch of sequences ends, another one takes its rows, and its pages move to the front of the pool

A case is a dict of plain values:
  kind              rotate | append | attend | fork | compact
  dtype             storage of queries, keys and values: f32 | bf16
  tokens, rot, interleaved, norm, first, scaling     rotate: rows; channels turned, pairs side by side or half of `rot` apart; whether
                    there is a norm; position of the first row; how frequencies are scaled for long contexts
  heads_q, heads, d heads of the queries, of keys and values, channels of a head
  seqs              sequences (fork: prompts, compact: of either batch)
  held, new         tokens a sequence holds before, and new ones
  ragged            whether sequences differ: held and new ones are then at most that, some have no new one
  block             tokens of a block, which is a page
  window, softcap, causal, lse    attend: keys in reach (0: all), bound of the scores (0: none), whether later keys are out of reach,
                    whether the logarithm of the sums is returned too
  beams             fork: continuations of a prompt
Sizes are those of the 2B-, 9B- and 27B-shaped layers of ``workloads`` and between them.
"""
from __future__ import annotations

import math

import torch

own = False
DEVICE = "cuda:0"
EPS = 1e-6
BASE = 10000.0
STRETCH, TRAINED = 8.0, 8192       # scaled frequencies: by how much, and the positions they were trained for
_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ----------------------------------------------------------------------------------------------------
# the cases
# ----------------------------------------------------------------------------------------------------
def _rotate(tokens, heads_q, heads, d, rot, dtype, interleaved, norm, first, scaling):
    return dict(kind="rotate", tokens=tokens, heads_q=heads_q, heads=heads, d=d, rot=rot, dtype=dtype, interleaved=interleaved, norm=norm,
                first=first, scaling=scaling)


def _append(seqs, new, held, ragged, heads, d, block, dtype):
    return dict(kind="append", seqs=seqs, new=new, held=held, ragged=ragged, heads=heads, d=d, block=block, dtype=dtype)


def _attend(seqs, new, held, ragged, heads_q, heads, d, block, dtype, window=0, softcap=0.0, causal=True, lse=False):
    return dict(kind="attend", seqs=seqs, new=new, held=held, ragged=ragged, heads_q=heads_q, heads=heads, d=d, block=block, dtype=dtype,
                window=window, softcap=softcap, causal=causal, lse=lse)


def _pages(kind, seqs, held, heads, d, block, beams=1):
    return dict(kind=kind, seqs=seqs, held=held, ragged=True, heads=heads, d=d, block=block, beams=beams)


def listed():
    return [
        # One decoded token of the 27B-shaped model: the smallest call.
        dict(name="rotate_1_27b", **_rotate(1, 32, 16, 128, 128, "bf16", False, True, 5000, "none")),
        # A prompt of the 9B-shaped model.
        dict(name="rotate_4096_9b", **_rotate(4096, 16, 8, 256, 256, "bf16", False, True, 0, "none")),
        # A ragged batch far into a long context, a quarter of each head turned, pairs side by side, no norm, float32.
        dict(name="rotate_333_part_f32", **_rotate(333, 10, 5, 80, 20, "f32", True, False, 1_000_000, "parts")),
        # Sixty-four sequences decoded together, one token each, into blocks that are partly filled.
        dict(name="append_64_27b", **_append(64, 1, 4000, True, 16, 128, 64, "bf16")),
        # A prompt of the 9B-shaped model behind a short prefix that ends inside a block.
        dict(name="append_8192_9b", **_append(1, 8192, 37, False, 8, 256, 64, "bf16")),
        # One token of one short sequence of the 2B-shaped model: what latency allows.
        dict(name="attend_1_2b", **_attend(1, 1, 511, False, 8, 4, 256, 64, "bf16", softcap=50.0)),
        # Forty-eight sequences of very different lengths decoded together, 27B-shaped: the largest cache.
        dict(name="attend_48_27b_long", **_attend(48, 1, 32767, True, 32, 16, 128, 64, "bf16")),
        # Three tokens each at once (drafts that are checked), sliding window, float32, small blocks, channels that fill no tile.
        dict(name="attend_24_window_f32", **_attend(24, 3, 5000, True, 10, 2, 80, 16, "f32", window=1000, lse=True)),
        # A prompt of the 9B-shaped model on its own.
        dict(name="attend_8192_9b", **_attend(1, 8192, 0, False, 16, 8, 256, 64, "bf16", softcap=50.0)),
        # Chunks of prompts and sequences with few or no new tokens in one batch, 27B-shaped, windowed, blocks of 32.
        dict(name="attend_mixed_27b", **_attend(17, 1500, 6000, True, 32, 16, 128, 32, "bf16", window=4096, lse=True)),
        # Four prompts with eight continuations each, at the step that forks them.
        dict(name="fork_4x8_27b", **_pages("fork", 4, 2000, 16, 128, 64, 8)),
        # A pool whose first half a finished batch has left.
        dict(name="compact_24_9b", **_pages("compact", 24, 8000, 8, 256, 64)),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(("rotate", "rotate", "append", "append", "attend", "attend", "attend", "attend", "fork", "compact"))
    heads = rng.choice((1, 2, 3, 4, 5, 8, 12, 16))
    heads_q = heads * rng.choice((1, 2, 2, 3, 4, 8))
    d = rng.choice((64, 128, 128, 256, 256, 16 * rng.randint(2, 16)))
    block = rng.choice((16, 32, 64, 64, 128))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    if kind == "rotate":
        tokens = _log_int(rng, 1, max(1, min(8192, 25_000_000 // ((heads_q + heads) * d))))
        rot = rng.choice((d, d, d // 2, 2 * rng.randint(1, d // 2)))
        return _rotate(tokens, heads_q, heads, d, rot, dtype, rng.random() < 0.4, rng.random() < 0.7, rng.choice((0, _log_int(rng, 1, 2_000_000))),
                       rng.choice(("none", "none", "linear", "base", "parts")))
    width = heads * d
    if kind == "append":
        seqs = _log_int(rng, 1, 64)
        new = rng.choice((1, 1, _log_int(rng, 1, max(1, min(8192, 16_000_000 // (seqs * width))))))
        return _append(seqs, new, _log_int(rng, 1, 2000), rng.random() < 0.7, heads, d, block, dtype)
    if kind == "attend":
        causal = rng.random() < 0.85
        extra = dict(window=rng.choice((0, 0, 0, _log_int(rng, 16, 4096))), softcap=rng.choice((0.0, 0.0, 30.0, 50.0)), causal=causal, lse=rng.random() < 0.3)
        ragged = rng.random() < 0.7
        if rng.random() < 0.5:      # few new tokens, the cache is what counts
            seqs, new = _log_int(rng, 1, 48), rng.choice((1, 1, 1, 2, 3, 5))
            held = _log_int(rng, 8, max(8, min(32767, 800_000_000 // (seqs * width))))
            return _attend(seqs, new, held, ragged, heads_q, heads, d, block, dtype, **extra)
        seqs = _log_int(rng, 1, 8)
        most = math.sqrt(1.2e11 / (seqs * heads_q * d * (2 if dtype == "f32" else 1)))       # tokens squared, as the largest prompt
        new = _log_int(rng, 8, max(8, min(8000, most)))
        return _attend(seqs, new, rng.choice((0, _log_int(rng, 1, max(1, min(8000, most ** 2 / new - new))))), ragged, heads_q, heads, d, block, dtype, **extra)
    seqs = _log_int(rng, 1, 24)
    held = _log_int(rng, 16, max(16, min(8000, 200_000_000 // (seqs * width))))
    return _pages(kind, seqs, held, heads, d, block, rng.randint(2, 8) if kind == "fork" else 1)


def _share(i, salt):
    """A number in [0, 1) that goes by the sequence alone."""
    return ((i + 1) * 2654435761 + salt * 40503 * 65537) % (1 << 32) / (1 << 32)


def _held(c):
    return [c["held"] if not c["ragged"] else int(c["held"] * (0.05 + 0.95 * _share(i, 1))) for i in range(c["seqs"])]


def _new(c):
    n = c["new"]
    if not c["ragged"] or n == 1:
        return [n] * c["seqs"]
    # some sequences bring few, some none
    got = [int((n + 1) * _share(i, 2) ** 3) for i in range(c["seqs"])]
    got[-1] = n
    return got


# ----------------------------------------------------------------------------------------------------
# inputs
# ----------------------------------------------------------------------------------------------------
def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEVICE)


def _starts(counts):
    at = [0]
    for n in counts:
        at.append(at[-1] + n)
    return at


def _heads(n, parts, d, dtype, gen, scales):
    """Views [n][heads][d] into one projection's output, as it leaves a fused product."""
    x = torch.randn((n, sum(parts) * d), generator=gen, device=DEVICE)
    views, at = [], 0
    for p, s in zip(parts, scales):
        part = x[:, at * d:(at + p) * d].view(n, p, d)
        part *= s
        part[:, :, torch.randperm(d, generator=gen, device=DEVICE)[:2]] *= 4.0       # channels that stand out in every token
        views.append((at, p))
        at += p
    x = x.to(dtype)
    return [x[:, a * d:(a + p) * d].view(n, p, d) for a, p in views]


def _fill(pages, heads, block, d, gen):
    """Codes [pages][heads][block][d] and scales [pages][heads] of Gaussian values with channels that stand out."""
    codes = torch.empty((pages, heads, block, d), dtype=torch.int8, device=DEVICE)
    scales = torch.empty((pages, heads), device=DEVICE)
    loud = torch.ones((heads, 1, d), device=DEVICE)
    loud[:, :, torch.randperm(d, generator=gen, device=DEVICE)[:2]] = 4.0
    step = max(1, 64_000_000 // (heads * block * d))
    for p in range(0, pages, step):
        x = torch.randn((min(step, pages - p), heads, block, d), generator=gen, device=DEVICE).mul_(loud)
        s = x.abs().amax((2, 3)) / 127.0
        codes[p:p + step] = x.div_(s[:, :, None, None]).round_()
        scales[p:p + step] = s
    return codes, scales


def _table(blocks, width, pages):
    """Rows of page numbers from the list `pages`, -1 behind a sequence's blocks."""
    at, rows = 0, []
    for b in blocks:
        rows.append(pages[at:at + b] + [-1] * (width - b))
        at += b
    return _ints(rows)


def _rotate_inputs(c, gen):
    q, k = _heads(c["tokens"], (c["heads_q"], c["heads"], c["heads"]), c["d"], _TYPES[c["dtype"]], gen, (3.0, 2.0, 1.0))[:2]
    s = {"q": q, "k": k, "positions": torch.arange(c["tokens"], device=DEVICE, dtype=torch.int32) + c["first"], "gain_q": None, "gain_k": None}
    if c["norm"]:
        s["gain_q"], s["gain_k"] = (torch.randn(c["d"], generator=gen, device=DEVICE) * 0.2 for _ in range(2))
    i = torch.arange(0, c["rot"], 2, dtype=torch.float64, device=DEVICE) / c["rot"]
    base = BASE * STRETCH ** (c["rot"] / max(1, c["rot"] - 2)) if c["scaling"] == "base" else BASE
    s["freq"], s["amplitude"] = base ** -i, 1.0
    if c["scaling"] == "linear":
        s["freq"] = s["freq"] / STRETCH
    elif c["scaling"] == "parts":
        keep = ((TRAINED * s["freq"] / (2 * math.pi) - 1.0) / (32.0 - 1.0)).clamp(0.0, 1.0)
        s["freq"], s["amplitude"] = s["freq"] * keep + s["freq"] / STRETCH * (1 - keep), 0.1 * math.log(STRETCH) + 1.0
    return s


def _cache_inputs(c, gen):
    """A pool whose pages are in any order, a twentieth of them of no sequence."""
    B, held, new = c["block"], _held(c), _new(c)
    lengths = [h + n for h, n in zip(held, new)]
    blocks = [-(-x // B) for x in lengths]
    pages = sum(blocks) + sum(blocks) // 20 + 1
    s = {"held": held, "new": new, "starts": _ints(_starts(new)), "lengths": _ints(lengths)}
    s["kc"], s["ks"] = _fill(pages, c["heads"], B, c["d"], gen)
    s["vc"], s["vs"] = _fill(pages, c["heads"], B, c["d"], gen)
    s["table"] = _table(blocks, max(blocks), torch.randperm(pages, generator=gen, device=DEVICE).tolist())
    s["refs"] = _held_by(s["table"], pages)
    if c["kind"] == "append":
        s["k"], s["v"] = _heads(sum(new), (2, c["heads"], c["heads"]), c["d"], _TYPES[c["dtype"]], gen, (1.0, 1.0, 1.0))[1:]
        # what is compared: all tokens of the blocks that the call writes to
        s["begin"] = [h // B * B if n else h + n for h, n in zip(held, new)]
        s["range"] = _starts([x - b for x, b in zip(lengths, s["begin"])])
    else:
        s["q"] = _heads(sum(new), (c["heads_q"], 1), c["d"], _TYPES[c["dtype"]], gen, (2.0, 1.0))[0]
    return s


def _held_by(table, pages):
    """How many rows hold each page."""
    return torch.bincount(table[table >= 0].long(), minlength=pages).to(torch.int32)


def _page_inputs(c, gen):
    B, held = c["block"], [max(1, x) for x in _held(c)]
    blocks = [-(-x // B) for x in held]
    used = sum(blocks)
    if c["kind"] == "fork":
        # prompts in the first rows, their continuations behind them: row i goes on from prompt i % seqs
        rows, width = c["seqs"] * c["beams"], max(blocks) + 1
        pages = used + 2 * rows + 3
        order = torch.randperm(pages, generator=gen, device=DEVICE).tolist()
        table = torch.full((rows, width), -1, dtype=torch.int32, device=DEVICE)
        table[:c["seqs"]] = _table(blocks, width, order)
        lengths = held + [0] * (rows - c["seqs"])
        sources = [i % c["seqs"] for i in range(rows)]
        counts = [0] * c["seqs"] + [1] * (rows - c["seqs"])
    else:
        # the batch that ends holds the first `used` pages, the one that takes over the rest but for the last ones, which are free
        rows, width = 2 * c["seqs"], max(blocks)
        pages = 2 * used + used // 10 + 1
        order = torch.randperm(used, generator=gen, device=DEVICE).tolist()
        table = torch.cat([_table(blocks, width, order), _table(blocks, width, list(range(used, 2 * used)))])
        lengths = held + held
        sources = [c["seqs"] + i for i in range(c["seqs"])] + [-1] * c["seqs"]
        counts = [0] * c["seqs"] + held      # the batch after that is given room at once
    s = {"table": table, "lengths": _ints(lengths), "refs": _held_by(table, pages), "sources": _ints(sources), "starts": _ints(_starts(counts)),
         "total": sum(counts)}
    s["kc"], s["ks"] = _fill(pages, c["heads"], B, c["d"], gen)
    s["vc"], s["vs"] = _fill(pages, c["heads"], B, c["d"], gen)
    return s


def _inputs(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(int(seed))
    kind = case["kind"]
    s = _rotate_inputs(case, gen) if kind == "rotate" else _page_inputs(case, gen) if kind in ("fork", "compact") else _cache_inputs(case, gen)
    s["case"] = dict(case)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        from paper_2511_19705_amd import cafeq
        if case["kind"] == "rotate":
            # the table of frequencies that a program makes once
            s["freq"], s["amplitude"] = cafeq.rotary_frequencies(case["rot"], base=BASE, scaling=case["scaling"], factor=STRETCH, trained=TRAINED, device=DEVICE)
            return s
        # the cache that a program holds
        kc = s.pop("kc")
        rows, width = s["table"].shape
        cache = cafeq.kv_cache(rows, kc.shape[0], kc.shape[1], kc.shape[3], block=kc.shape[2], width=width, device=DEVICE)
        cache.k.copy_(kc)
        cache.v.copy_(s.pop("vc").transpose(2, 3))
        for t, name in ((cache.kscale, "ks"), (cache.vscale, "vs"), (cache.table, "table"), (cache.lengths, "lengths"), (cache.refs, "refs")):
            t.copy_(s.pop(name))
        s["cache"] = cache
        if case["kind"] == "append":
            s["begin"] = _ints(s["begin"])
            s["total"] = s["range"][-1]
            s["range"] = _ints(s["range"])
    return s


# ----------------------------------------------------------------------------------------------------
# one pass: the plain forms
# ----------------------------------------------------------------------------------------------------
def _plain_turn(x, gain, s):
    c = s["case"]
    y = x.float()
    if c["norm"]:
        y = y * torch.rsqrt(y.square().mean(2, keepdim=True) + EPS) * (1.0 + gain)
    angle = s["positions"].double()[:, None] * s["freq"]          # 32 bits lose the angles of far positions
    cos, sin = ((f(angle) * s["amplitude"]).float()[:, None, :] for f in (torch.cos, torch.sin))
    r = c["rot"]
    if c["interleaved"]:
        a, b = y[:, :, 0:r:2], y[:, :, 1:r:2]
        turned = torch.stack((a * cos - b * sin, a * sin + b * cos), 3).flatten(2)
    else:
        a, b = y[:, :, :r // 2], y[:, :, r // 2:r]
        turned = torch.cat((a * cos - b * sin, a * sin + b * cos), 2)
    return torch.cat((turned, y[:, :, r:]), 2).to(x.dtype)


def _places(s, begin, counts):
    """(page, place in it) of `counts` tokens a sequence from `begin` on."""
    n = _ints(counts).long()
    row = torch.repeat_interleave(torch.arange(len(counts), device=DEVICE), n)
    first = torch.cumsum(n, 0) - n
    pos = torch.arange(row.numel(), device=DEVICE) - first[row] + _ints(begin).long()[row]
    B = s["case"]["block"]
    return s["table"][row, pos // B].long(), pos % B


def _plain_store(x, codes, scales, page, slot, open_page, open_used):
    """New tokens x at (page, slot); open_page: the blocks that held open_used tokens before."""
    x = x.float()
    top = torch.zeros_like(scales).scatter_reduce_(0, page[:, None].expand(-1, x.shape[1]), x.abs().amax(2), "amax") / 127.0
    old = scales[open_page].clone()
    scales[page] = top[page]
    scales[open_page] = torch.maximum(old, top[open_page])
    now = scales[open_page]
    held = codes[open_page].float() * torch.where(now > 0, old / now, torch.ones_like(now))[:, :, None, None]
    keep = torch.arange(codes.shape[2], device=DEVICE)[None, :] < open_used[:, None]
    codes[open_page] = torch.where(keep[:, None, :, None], torch.round(held).to(torch.int8), codes[open_page])
    inv = torch.where(scales > 0, 1.0 / scales, torch.zeros_like(scales))[page]
    codes[page, :, slot] = torch.round(x * inv[:, :, None]).clamp_(-127, 127).to(torch.int8)


def _plain_append(s):
    c, B = s["case"], s["case"]["block"]
    page, slot = _places(s, s["held"], s["new"])
    held, new = _ints(s["held"]).long(), _ints(s["new"]).long()
    open_rows = ((held % B > 0) & (new > 0)).nonzero()[:, 0]
    open_page, used = s["table"][open_rows, held[open_rows] // B].long(), held[open_rows] % B
    _plain_store(s["k"], s["kc"], s["ks"], page, slot, open_page, used)
    _plain_store(s["v"], s["vc"], s["vs"], page, slot, open_page, used)
    page, slot = _places(s, s["begin"], [b - a for a, b in zip(s["range"], s["range"][1:])])
    k = (s["kc"][page, :, slot].float() * s["ks"][page][:, :, None]).to(torch.bfloat16)
    v = (s["vc"][page, :, slot].float() * s["vs"][page][:, :, None]).to(torch.bfloat16)
    return {"k": k, "v": v, "kscale": s["ks"], "vscale": s["vs"]}


def _reach(c, held, new):
    """First and last + 1 key that any of a sequence's new tokens reaches."""
    return max(0, held - c["window"] + 1) if c["window"] else 0, held + new


def _masked(c, held, n, lo, hi):
    """[n][hi - lo]: keys out of reach."""
    at = torch.arange(held, held + n, device=DEVICE)[:, None]
    key = torch.arange(lo, hi, device=DEVICE)[None, :]
    out = torch.zeros((n, hi - lo), dtype=torch.bool, device=DEVICE)
    if c["causal"]:
        out |= key > at
    if c["window"]:
        out |= key <= at - c["window"]
    return out


def _plain_keys(s, row, lo, hi, codes, scales):
    """Values [heads][keys][d] of a row's tokens lo .. hi."""
    B = s["case"]["block"]
    first = lo // B
    page = s["table"][row, first:-(-hi // B)].long()
    x = codes[page].float() * scales[page][:, :, None, None]
    return x.transpose(0, 1).flatten(1, 2)[:, lo - first * B:hi - first * B]


def _plain_attend(s):
    c = s["case"]
    h, hq, d = c["heads"], c["heads_q"], c["d"]
    out = torch.empty((s["q"].shape[0], hq, d), dtype=s["q"].dtype, device=DEVICE)
    lse = torch.empty((s["q"].shape[0], hq), device=DEVICE)
    at = 0
    for row, (held, n) in enumerate(zip(s["held"], s["new"])):       # sequences differ: padded to one length they would cost several times as much
        if n == 0:
            continue
        lo, hi = _reach(c, held, n)
        q = s["q"][at:at + n].float().transpose(0, 1).reshape(h, -1, d)         # heads that share keys behind each other
        x = torch.matmul(q, _plain_keys(s, row, lo, hi, s["kc"], s["ks"]).transpose(1, 2).contiguous()).mul_(d ** -0.5)
        if c["softcap"]:
            x = x.div_(c["softcap"]).tanh_().mul_(c["softcap"])
        if c["causal"] and n > 1 or c["window"]:
            x = x.view(h, hq // h, n, hi - lo).masked_fill_(_masked(c, held, n, lo, hi), -math.inf).view(h, -1, hi - lo)
        top = x.amax(2, keepdim=True)
        x = x.sub_(top).exp_()
        total = x.sum(2, keepdim=True)
        y = torch.matmul(x, _plain_keys(s, row, lo, hi, s["vc"], s["vs"]).contiguous()) / total
        out[at:at + n] = y.view(hq, n, d).transpose(0, 1).to(out.dtype)
        lse[at:at + n] = (top + torch.log(total)).view(hq, n).t()
        at += n
    return {"out": out, "lse": lse} if c["lse"] else {"out": out}


def _plain_reorder(s):
    take = s["sources"].long()
    there = take >= 0
    s["table"] = torch.where(there[:, None], s["table"][take.clamp(min=0)], -1).to(torch.int32)
    s["lengths"] = torch.where(there, s["lengths"][take.clamp(min=0)], 0).to(torch.int32)
    s["refs"] = _held_by(s["table"], s["refs"].numel())


def _plain_reserve(s):
    """Room for the new tokens: shared blocks that are appended to are copied, missing ones taken from the lowest free pages, row by row.
    Returns the new tokens' positions."""
    B, rows = s["case"]["block"], s["table"].shape[0]
    new = (s["starts"][1:] - s["starts"][:-1]).long()
    length = s["lengths"].long()
    have, need = -(-length // B), -(-(length + new) // B)
    last = s["table"][torch.arange(rows, device=DEVICE), (have - 1).clamp(min=0)].long()
    copied = (length % B > 0) & (new > 0) & (s["refs"][last.clamp(min=0)] > 1)
    count = need - have + copied.long()
    row = torch.repeat_interleave(torch.arange(rows, device=DEVICE), count)
    nth = torch.arange(row.numel(), device=DEVICE) - (torch.cumsum(count, 0) - count)[row]
    free = (s["refs"] == 0).nonzero()[:row.numel(), 0].to(torch.int32)
    s["table"][row, have[row] - copied.long()[row] + nth] = free
    to = s["table"][torch.arange(rows, device=DEVICE), (have - 1).clamp(min=0)].long()[copied]
    for t in (s["kc"], s["vc"], s["ks"], s["vs"]):
        t[to] = t[last[copied]]
    s["refs"] = _held_by(s["table"], s["refs"].numel())
    s["lengths"] = (length + new).to(torch.int32)
    row = torch.repeat_interleave(torch.arange(rows, device=DEVICE), new)
    return (torch.arange(row.numel(), device=DEVICE) - s["starts"].long()[row] + length[row]).to(torch.int32)


def _plain_compact(s):
    used = s["refs"] > 0
    count = used.sum()
    number = torch.arange(used.numel(), device=DEVICE)
    src, dst = (used & (number >= count)).nonzero()[:, 0], (~used & (number < count)).nonzero()[:, 0]
    for t in (s["kc"], s["vc"], s["ks"], s["vs"]):
        t[dst] = t[src]
    to = number.to(torch.int32)
    to[src] = dst.to(torch.int32)
    s["table"] = torch.where(s["table"] >= 0, to[s["table"].clamp(min=0).long()], s["table"])
    s["refs"] = _held_by(s["table"], s["refs"].numel())
    return count.to(torch.int32).view(1)


def _run_plain(s):
    kind = s["case"]["kind"]
    if kind == "rotate":
        return {"q": _plain_turn(s["q"], s["gain_q"], s), "k": _plain_turn(s["k"], s["gain_k"], s)}
    if kind == "append":
        return _plain_append(s)
    if kind == "attend":
        return _plain_attend(s)
    _plain_reorder(s)
    if kind == "fork":
        # rows that continued a prompt before are let go by the same call, so that a pass leaves what it found
        r = {"positions": _plain_reserve(s)}
    else:
        r = {"used": _plain_compact(s), "positions": _plain_reserve(s)}
    # pages are copied, not computed: their codes are compared as they are
    return {**r, "table": s["table"], "lengths": s["lengths"], "refs": s["refs"], "k": s["kc"], "v": s["vc"], "kscale": s["ks"], "vscale": s["vs"]}


# ----------------------------------------------------------------------------------------------------
# one pass: the framework's calls
# ----------------------------------------------------------------------------------------------------
def _run_own(s):
    from paper_2511_19705_amd import cafeq
    c = s["case"]
    kind = c["kind"]
    if kind == "rotate":
        q, k = cafeq.rotate_heads(s["q"], s["k"], s["positions"], s["freq"], interleaved=c["interleaved"], norm=c["norm"], gain_q=s["gain_q"],
                                  gain_k=s["gain_k"], eps=EPS, gain_offset=1.0, amplitude=s["amplitude"])
        return {"q": q, "k": k}
    cache = s["cache"]
    if kind == "append":
        cafeq.cache_append(cache, s["k"], s["v"], s["starts"], longest=max(s["new"]))
        k, v = cafeq.cache_values(cache, s["begin"], s["range"], s["total"], dtype=torch.bfloat16)
        return {"k": k, "v": v, "kscale": cache.kscale, "vscale": cache.vscale}
    if kind == "attend":
        r = cafeq.cache_attend(cache, s["q"], s["starts"], longest=max(s["new"]), window=c["window"], softcap=c["softcap"], causal=c["causal"], lse=c["lse"])
        return {"out": r[0], "lse": r[1]} if c["lse"] else {"out": r}
    cafeq.cache_reorder(cache, s["sources"])
    r = {} if kind == "fork" else {"used": cafeq.cache_compact(cache)}
    r["positions"] = cafeq.cache_reserve(cache, s["starts"], s["total"]).positions
    return {**r, "table": cache.table, "lengths": cache.lengths, "refs": cache.refs, "k": cache.k, "v": cache.v.transpose(2, 3), "kscale": cache.kscale,
            "vscale": cache.vscale}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ----------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ----------------------------------------------------------------------------------------------------
def _exact_turn(x, gain, s):
    c = s["case"]
    y = x.double()
    if c["norm"]:
        y = y / torch.sqrt((y * y).sum(2, keepdim=True) / c["d"] + EPS) * (1.0 + gain.double())
    out, half = y.clone(), c["rot"] // 2
    for i in range(half):
        p, q = (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + half)
        angle = (s["positions"].double() * s["freq"][i])[:, None]
        out[:, :, p] = s["amplitude"] * (y[:, :, p] * torch.cos(angle) - y[:, :, q] * torch.sin(angle))
        out[:, :, q] = s["amplitude"] * (y[:, :, p] * torch.sin(angle) + y[:, :, q] * torch.cos(angle))
    return out


def _exact_pages(x, codes, scales, held, new, begin, row, block, table):
    """A sequence's tokens from `begin` on, [tokens][heads][d]; scales are updated."""
    got = []
    for b in range(begin // block, -(-(held + new) // block)) if new else ():
        page = int(table[row][b])
        first, last = max(held, b * block), min(held + new, (b + 1) * block)
        old = codes[page, :, :max(0, held - b * block)].double()
        fresh = x[first - held:last - held].double()
        s = fresh.abs().amax((0, 2)) / 127.0
        if old.shape[1]:
            before = scales[page]
            s = torch.maximum(s, before)
            old = torch.round(old * (before / s)[:, None, None])
        scales[page] = s
        fresh = torch.round(fresh / torch.where(s > 0, s, torch.ones_like(s))[None, :, None])
        got.append(torch.cat((old.transpose(0, 1), fresh)) * s[None, :, None])
    return torch.cat(got) if got else x[:0].double()


def _exact_append(s):
    c, table = s["case"], s["table"].tolist()
    r = {"kscale": s["ks"].double(), "vscale": s["vs"].double()}
    for name, codes in (("k", s["kc"]), ("v", s["vc"])):
        at, rows = 0, []
        for row, (held, n) in enumerate(zip(s["held"], s["new"])):
            rows.append(_exact_pages(s[name][at:at + n], codes, r[name + "scale"], held, n, s["begin"][row], row, c["block"], table))
            at += n
        r[name] = torch.cat(rows)
    return r


def _exact_attend(s):
    c = s["case"]
    h, hq, d, B = c["heads"], c["heads_q"], c["d"], c["block"]
    n_all = s["q"].shape[0]
    out, lse = torch.empty((n_all, hq, d), dtype=torch.float64, device=DEVICE), torch.empty((n_all, hq), dtype=torch.float64, device=DEVICE)
    at = 0
    for row, (held, n) in enumerate(zip(s["held"], s["new"])):
        if not n:
            continue
        lo, hi = _reach(c, held, n)
        page = s["table"][row, :-(-hi // B)].long()
        mask = _masked(c, held, n, lo, hi)
        for g in range(h):
            K = (s["kc"][page, g].double() * s["ks"][page, g].double()[:, None, None]).reshape(-1, d)[lo:hi]
            V = (s["vc"][page, g].double() * s["vs"][page, g].double()[:, None, None]).reshape(-1, d)[lo:hi]
            for j in range(g * (hq // h), (g + 1) * (hq // h)):
                x = s["q"][at:at + n, j].double() @ K.t() / math.sqrt(d)
                if c["softcap"]:
                    x = c["softcap"] * torch.tanh(x / c["softcap"])
                x[mask] = -math.inf
                norm = torch.logsumexp(x, 1)
                out[at:at + n, j] = torch.exp(x - norm[:, None]) @ V
                lse[at:at + n, j] = norm
        at += n
    return {"out": out, "lse": lse} if c["lse"] else {"out": out}


def exact(case, seed):
    s = _inputs(case, seed)
    if case["kind"] == "rotate":
        return {"q": _exact_turn(s["q"], s["gain_q"], s), "k": _exact_turn(s["k"], s["gain_k"], s)}
    if case["kind"] == "append":
        return _exact_append(s)
    return _exact_attend(s) if case["kind"] == "attend" else None


# ----------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ----------------------------------------------------------------------------------------------------
def _keys_in_reach(c, held, n):
    """Keys of all new tokens of a sequence together."""
    total = 0
    for p in range(held, held + n):
        hi = p + 1 if c["causal"] else held + n
        total += hi - (max(0, p - c["window"] + 1) if c["window"] else 0)
    return total


def work(case):
    c = case
    size = 4 if c.get("dtype") == "f32" else 2
    if c["kind"] == "rotate":
        n = c["tokens"] * (c["heads_q"] + c["heads"])
        return {"bytes": float(2 * size * n * c["d"] + 4 * c["tokens"] + 4 * c["rot"]), "flops": float(n * (4 * c["d"] * c["norm"] + 3 * c["rot"]))}
    held = _held(c)
    width, B = c["heads"] * c["d"], c["block"]
    if c["kind"] == "append":
        new = _new(c)
        opened = sum(h % B for h, n in zip(held, new) if n)
        n, blocks = sum(new), sum(-(-(h % B + m) // B) for h, m in zip(held, new) if m)
        # read and write codes of open blocks; values in, codes out; codes of all blocks written to read back as bfloat16
        return {"bytes": float(2 * width * (2 * opened + n * (size + 1) + 3 * (n + opened)) + 16 * blocks * c["heads"]), "flops": float(4 * width * (n + opened))}
    if c["kind"] == "attend":
        new = _new(c)
        keys = sum(hi - lo for lo, hi in (_reach(c, h, n) for h, n in zip(held, new) if n))
        q = sum(new) * c["heads_q"]
        reach = sum(_keys_in_reach(c, h, n) for h, n in zip(held, new))
        return {"bytes": float(2 * width * keys + 8 * c["heads"] * (keys // B) + 2 * size * q * c["d"]), "flops": float(4 * c["d"] * c["heads_q"] * reach)}
    page = 2 * B * width + 8 * c["heads"]
    blocks = [-(-max(1, h) // B) for h in held]
    entries = 2 * 4 * sum(blocks) * (c["beams"] if c["kind"] == "fork" else 2)
    copies = (c["beams"] - 1) * sum(1 for h in held if max(1, h) % B) if c["kind"] == "fork" else sum(blocks)
    return {"bytes": float(2 * copies * page + entries), "flops": 0.0}
