"""GPU parity: attention over the 8-bit cache (cafeq_cache_attend) against float64 on the same codes and scales.

Tolerance, from the arithmetic, u = 2^-24.  A row's scores are sums over d channels: queries of bfloat16 and codes are exact, a float32 query is
taken in two parts of 11 bits that leave 2^-22 of it; with d products, in two parts each, accumulated in float32
    |x - ref| <= ((2 d + 8) u + 2^-22) size + 8 u |x|,     size = the largest scale sum_c |q K| of the row
(8 u: products with the scales, soft cap, the exponent's argument; the cap passes errors on at most as they are).  A weight exp(x - max) is
therefore off by e = 2 (that bound with |x| <= size) + 4 u of itself, numerator and denominator, and rounded to 11 bits (2^-12) with bfloat16,
in two parts (2^-22) with float32.  The sum over N keys adds N u.  With W = sum p |V|
    |out - ref| <= (2 e + r + (N + 16) u) W + h |out| + 2^-38 floor,     r = 2^-12 or 2^-22, h = 2^-8 for results of bfloat16
    |lse - ref| <= 2 e + (N + 16) u + 8 u |lse|
Weights p mant < 2^15 (p 2^14 at most, M rounded up by less than 1) below 2^-14 are subnormal in float16 and off by 2^-25 at most each, in the
numerator sum p mant c of out = sum p mant c / sum p 2^-exp; the denominator is above 2^13 2^-exp of the key with the largest y, and 2^exp <= vs:
    2^-25 sum |c| / (2^13 2^-exp) <= 2^-38 sum |c| max vs     more for out, "floor" below
and, errors being of either sign, 3e-6 (float32) or 2^-8 (bfloat16) of the 2-norm of W."""
import math

import numpy as np
import pytest

from tests import cache_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2511_19705_amd import cafeq
    return torch, cafeq


def _cache(env, lengths, heads, d, block, seed=0, spare=3, width=None):
    """A cache of random codes and scales that differ from page to page, pages in any order."""
    torch, cafeq = env
    gen = torch.Generator(device="cuda:0").manual_seed(seed)
    blocks = [-(-x // block) for x in lengths]
    pages = sum(blocks) + spare
    width = max(blocks + [1]) if width is None else width
    cache = cafeq.kv_cache(len(lengths), pages, heads, d, block=block, width=width)
    cache.k.copy_(torch.randn(cache.k.shape, generator=gen, device="cuda:0").mul_(40).clamp_(-127, 127))
    cache.v.copy_(torch.randn(cache.v.shape, generator=gen, device="cuda:0").mul_(40).clamp_(-127, 127))
    cache.kscale.copy_(torch.exp(torch.randn(cache.kscale.shape, generator=gen, device="cuda:0") * 0.4 - 3.7))
    cache.vscale.copy_(torch.exp(torch.randn(cache.vscale.shape, generator=gen, device="cuda:0") * 0.7 - 3.7))
    order = torch.randperm(pages, generator=gen, device="cuda:0").to(torch.int32)
    at = 0
    for i, b in enumerate(blocks):
        cache.table[i, :b] = order[at:at + b]
        at += b
    cache.lengths.copy_(torch.tensor(lengths, dtype=torch.int32))
    return cache


def _starts(counts, lead=0):
    s = [lead]
    for c in counts:
        s.append(s[-1] + c)
    return s


def _near(env, cache, q, starts, out, lse, scale=None, softcap=0.0, window=0, causal=True):
    torch = env[0]
    d = q.shape[2]
    want, wlse, W, size, floor = R.attend(torch, cache, q, starts, d ** -0.5 if scale is None else scale, softcap, window, causal)
    rows = slice(starts[0], starts[-1])
    out, want, W, size, wlse, floor = out[rows].double(), want[rows], W[rows], size[rows], wlse[rows], floor[rows]
    u, f32 = 2.0 ** -24, q.dtype == torch.float32
    N = int(cache.lengths.max())
    e = 2 * (((2 * d + 16) * u + 2.0 ** -22) * size) + 4 * u
    tol = (2 * e + (2.0 ** -22 if f32 else 2.0 ** -12) + (N + 16) * u)[:, :, None] * W + (0 if f32 else 2.0 ** -8) * want.abs() + 2.0 ** -38 * floor + 1e-37
    err = (out - want).abs()
    assert not torch.isnan(err).any()
    assert (err <= tol).all(), float((err / tol).max())
    assert float(err.norm()) <= (3e-6 if f32 else 2.0 ** -8) * float(W.norm()) + 1e-30
    if lse is not None:
        got = lse[rows].double()
        none = torch.isneginf(wlse)
        assert torch.equal(torch.isneginf(got), none)
        diff = (got - wlse)[~none].abs()
        assert (diff <= (2 * e + (N + 16) * u + 8 * u * wlse.abs())[~none]).all()


def _run(env, counts, lengths, hq, h, d, block, dtype, seed=0, lead=0, tail=0, fused=True, given_out=False, longest=None, cache=None, **kw):
    torch, cafeq = env
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    cache = _cache(env, lengths, h, d, block, seed) if cache is None else cache
    gen = torch.Generator(device="cuda:0").manual_seed(seed + 1)
    starts = _starts(counts, lead)
    n = starts[-1] + tail
    x = (torch.randn((n, (hq + (8 if fused else 0)) * d), generator=gen, device="cuda:0") * 2).to(t)
    q = x[:, :hq * d].unflatten(1, (hq, d))
    out = torch.full((n, hq, d), 7.0, dtype=t, device="cuda:0") if given_out or lead or tail else None
    s = torch.tensor(starts, dtype=torch.int32, device="cuda:0")
    got, lse = cafeq.cache_attend(cache, q, s, lse=True, out=out, longest=longest, **kw)
    assert torch.equal(got, cafeq.cache_attend(cache, q, s, longest=longest, out=None if out is None else torch.full_like(out, 7.0), **kw))
    _near(env, cache, q, starts, got, lse, **kw)
    if out is not None:
        assert (out[:lead] == 7.0).all() and (out[n - tail:] == 7.0).all()
    return cache, q, s, got, lse


DIMS = [16, 32, 48, 64, 80, 128, 144, 192, 208, 256]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", DIMS)
@pytest.mark.parametrize("block", [16, 32, 64, 128])
def test_single_tokens(env, dtype, d, block):
    _run(env, [1, 1, 1, 1, 1, 1], [1, 15, 64, 65, 300, 1000], 4, 2, d, block, dtype, seed=d, longest=1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,h", [(1, 1), (3, 1), (8, 8), (8, 1), (16, 1), (20, 4), (34, 2), (64, 1)])
def test_shared_heads(env, dtype, hq, h):
    for counts in ([1, 1, 1], [2, 5, 1], [40, 0, 17]):
        _run(env, counts, [70, 333, 129], hq, h, 64, 32, dtype, seed=hq)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", DIMS)
def test_prompts(env, dtype, d):
    _run(env, [200, 1, 0, 65], [200, 1, 77, 400], 4, 2, d, 64, dtype, seed=d)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("block", [16, 32, 64, 128])
@pytest.mark.parametrize("window", [0, 1, 5, 64, 100, 1000])
@pytest.mark.parametrize("causal", [True, False])
def test_windows(env, dtype, block, window, causal):
    _run(env, [130, 3, 1, 16], [300, 3, 500, 16], 4, 2, 64, block, dtype, window=window, causal=causal)
    _run(env, [1, 2, 1], [300, 3, 500], 4, 2, 64, block, dtype, window=window, causal=causal)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("softcap,scale", [(0.0, 1.0), (50.0, None), (3.0, 0.5), (1.0, -0.3), (0.0, 0.0)])
def test_scores(env, dtype, softcap, scale):
    for counts, lengths in (([90, 1], [200, 700]), ([1, 1], [200, 700])):
        _run(env, counts, lengths, 4, 4, 128, 64, dtype, softcap=softcap, scale=scale)


@pytest.mark.parametrize("counts,lengths", [([1], [5000]), ([1], [40000]), ([3], [20000]), ([40], [20000]), ([1, 1], [1, 30000]), ([700], [700]), ([513], [9000]),
                                            ([1] * 70, [17 * i + 1 for i in range(70)]), ([300, 1, 1, 1, 1, 1, 40], [300, 6000, 1, 90, 4000, 12000, 2000])])
def test_lengths(env, counts, lengths):
    for dtype in ("bf16", "f32"):
        _run(env, counts, lengths, 4, 2, 128, 64, dtype)


def test_rows_of_no_sequence_are_left(env):
    for dtype in ("bf16", "f32"):
        for counts in ([1, 1, 0, 1], [50, 3, 0, 200]):
            _run(env, counts, [60, 100, 5, 300], 4, 2, 80, 32, dtype, lead=3, tail=4)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_without_keys(env, dtype):
    torch, cafeq = env
    # more rows than tokens: the first ones stand before the beginning; an empty sequence
    for counts in ([5, 2, 1], [90, 70, 1]):
        for causal in (True, False):
            _, _, _, out, lse = _run(env, counts, [3, 0, 40], 4, 2, 64, 16, dtype, causal=causal)
            first = counts[0] if not causal else counts[0] - 3
            assert (out[counts[0]:counts[0] + counts[1]] == 0).all() and torch.isneginf(lse[counts[0]:counts[0] + counts[1]]).all()
            if causal:
                assert (out[:first] == 0).all() and torch.isneginf(lse[:first]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("block", [16, 128])
def test_pages_that_are_not_there_are_no_keys(env, dtype, block):
    torch, _ = env
    for counts in ([1, 1, 1], [100, 1, 20]):
        cache = _cache(env, [300, 300, 20], 2, 64, block)
        cache.table[0, 1], cache.table[1, 0], cache.table[2, 0] = -1, cache.k.shape[0], -2 ** 31
        if block == 128:
            cache.table[1, 1:] = 2 ** 31 - 1
        cache.kscale[0], cache.vscale[0] = float("nan"), float("nan")      # what a clamped number would read
        used = set(cache.table.flatten().tolist())
        if 0 in used:
            i, b = (cache.table == 0).nonzero()[0].tolist()
            cache.table[i, b] = next(p for p in range(cache.k.shape[0]) if p not in used)
        _run(env, counts, [300, 300, 20], 4, 2, 64, block, dtype, cache=cache)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_what_is_out_of_reach_has_no_effect(env, dtype, bad):
    """Scales that are no numbers and codes of any kind behind the length, behind the window and in other sequences' pages."""
    torch, cafeq = env
    for counts in ([1, 1], [70, 2]):
        cache = _cache(env, [500, 200], 2, 64, 64)
        starts = torch.tensor(_starts(counts), dtype=torch.int32, device="cuda:0")
        q = torch.randn((sum(counts), 4, 64), device="cuda:0").to(torch.float32 if dtype == "f32" else torch.bfloat16)
        want = cafeq.cache_attend(cache, q, starts, window=100, lse=True)
        reach = set(cache.table[0, (500 - counts[0] - 99) // 64:8].tolist() + cache.table[1, (200 - counts[1] - 99) // 64:4].tolist())
        for p in range(cache.k.shape[0]):
            if p not in reach:
                cache.kscale[p], cache.vscale[p] = bad, bad
        last = int(cache.table[1, 3])
        cache.k[last, :, 8:], cache.v[last, :, :, 8:] = -128, 127
        got = cafeq.cache_attend(cache, q, starts, window=100, lse=True)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        # later keys, in a page of their own, do not reach earlier rows
        if counts[0] > 60:
            cache.kscale[cache.table[0, 7]], cache.vscale[cache.table[0, 7]] = bad, bad
            got = cafeq.cache_attend(cache, q, starts, window=100)
            inside = counts[0] - (500 - 448)
            assert torch.equal(got[:inside], want[0][:inside]) and torch.isnan(got[inside:counts[0]]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("side", ["kscale", "vscale"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_scales_that_are_no_numbers_show(env, dtype, side, bad):
    torch, cafeq = env
    for counts in ([1, 1], [70, 2]):
        cache = _cache(env, [500, 200], 2, 64, 64)
        starts = torch.tensor(_starts(counts), dtype=torch.int32, device="cuda:0")
        q = torch.randn((sum(counts), 4, 64), device="cuda:0").to(torch.float32 if dtype == "f32" else torch.bfloat16)
        want = cafeq.cache_attend(cache, q, starts)
        getattr(cache, side)[cache.table[0, 3], 1] = bad
        cache.k[cache.table[0, 3], 1] = 0
        cache.v[cache.table[0, 3], 1] = 0
        got = cafeq.cache_attend(cache, q, starts)
        assert torch.isnan(got[:counts[0], 2:]).all()
        assert torch.equal(got[:counts[0], :2], want[:counts[0], :2]) and torch.equal(got[counts[0]:], want[counts[0]:])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_queries_that_are_no_numbers_stay_in_their_row(env, dtype, bad):
    torch, cafeq = env
    for counts in ([1, 3], [70, 2]):
        cache = _cache(env, [500, 200], 2, 64, 64)
        starts = torch.tensor(_starts(counts), dtype=torch.int32, device="cuda:0")
        q = torch.randn((sum(counts), 4, 64), device="cuda:0").to(torch.float32 if dtype == "f32" else torch.bfloat16)
        want = cafeq.cache_attend(cache, q, starts)
        q[counts[0] + 1, 2, 5] = bad
        got = cafeq.cache_attend(cache, q, starts)
        assert torch.isnan(got[counts[0] + 1, 2]).all()
        got[counts[0] + 1, 2] = want[counts[0] + 1, 2]
        assert torch.equal(got, want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_magnitudes(env, dtype):
    """Scales of v from page to page over many decades, pages of zeros, queries far from one, scores that leave one key."""
    torch, _ = env
    for counts, lengths in (([1, 1, 1], [900, 64, 300]), ([100, 64, 20], [900, 64, 300])):
        cache = _cache(env, lengths, 2, 64, 64)
        cache.vscale.copy_(10.0 ** torch.linspace(-12, 12, cache.vscale.numel(), device="cuda:0").view(cache.vscale.shape))
        _run(env, counts, lengths, 4, 2, 64, 64, dtype, cache=cache)
        for p in cache.table[0, ::3].tolist():
            cache.v[p], cache.vscale[p] = 0, 0.0
        _run(env, counts, lengths, 4, 2, 64, 64, dtype, cache=cache)
        cache.v.zero_()
        cache.vscale.zero_()
        out = _run(env, counts, lengths, 4, 2, 64, 64, dtype, cache=cache)[3]
        assert (out == 0).all()
        cache = _cache(env, lengths, 2, 64, 64)
        cache.kscale.mul_(1e6)
        _run(env, counts, lengths, 4, 2, 64, 64, dtype, cache=cache, scale=1e-5)
        cache.kscale.mul_(1e-20)
        _run(env, counts, lengths, 4, 2, 64, 64, dtype, cache=cache, scale=1e13)


def test_layouts_of_q_and_out(env):
    torch, cafeq = env
    for dtype in (torch.float32, torch.bfloat16):
        for counts in ([1, 1], [3, 90]):
            cache = _cache(env, [100, 300], 2, 64, 32)
            n = sum(counts)
            starts = torch.tensor(_starts(counts), dtype=torch.int32, device="cuda:0")
            q = torch.randn((n, 4, 64), device="cuda:0").to(dtype)
            want = cafeq.cache_attend(cache, q, starts)
            first = q.transpose(0, 1).contiguous().transpose(0, 1)
            assert torch.equal(cafeq.cache_attend(cache, first, starts), want)
            out = torch.full((4, n, 96), 3.0, device="cuda:0", dtype=dtype)
            assert cafeq.cache_attend(cache, first, starts, out=out[:, :, 16:80].transpose(0, 1)).data_ptr() == out[:, :, 16:80].data_ptr()
            assert torch.equal(out[:, :, 16:80].transpose(0, 1), want) and (out[:, :, :16] == 3).all() and (out[:, :, 80:] == 3).all()
            both = torch.cat((q, torch.zeros_like(q)), 1)       # q and the result in turn within each row
            cafeq.cache_attend(cache, both[:, :4], starts, out=both[:, 4:])
            assert torch.equal(both[:, 4:], want) and torch.equal(both[:, :4], q)


@pytest.mark.parametrize("longest", [1, 2, 20, 64])
def test_rows_beyond_the_bound_are_left(env, longest):
    torch, cafeq = env
    counts = [70, 1, 25]
    cache = _cache(env, [200, 300, 25], 2, 64, 32)
    starts = torch.tensor(_starts(counts), dtype=torch.int32, device="cuda:0")
    q = torch.randn((96, 4, 64), device="cuda:0").bfloat16()
    want = cafeq.cache_attend(cache, q, starts)
    got = cafeq.cache_attend(cache, q, starts, longest=longest, out=torch.full_like(want, 7.0))
    at = 0
    for c in counts:
        near = (got[at:at + min(c, longest)].float() - want[at:at + min(c, longest)].float()).abs() <= 2.0 ** -6 * (want[at:at + min(c, longest)].float().abs() + 0.5)
        assert near.all() and (got[at + min(c, longest):at + c] == 7.0).all()
        at += c


def test_streams_and_calls_at_once(env):
    torch, cafeq = env
    jobs = []
    for i, (counts, lengths) in enumerate((([1] * 8, [4000] * 8), ([300, 1], [300, 9000]), ([2] * 5, [700] * 5), ([64], [12000]))):
        cache = _cache(env, lengths, 2, 128, 64, seed=i)
        q = torch.randn((sum(counts), 8, 128), device="cuda:0").bfloat16()
        s = torch.tensor(_starts(counts), dtype=torch.int32, device="cuda:0")
        jobs.append((cache, q, s, cafeq.cache_attend(cache, q, s)))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in jobs]
    got = [[] for _ in jobs]
    for _ in range(10):
        for j, (cache, q, s, _) in enumerate(jobs):
            with torch.cuda.stream(streams[j]):
                got[j].append(cafeq.cache_attend(cache, q, s))
    torch.cuda.synchronize()
    for (_, _, _, want), outs in zip(jobs, got):
        assert all(torch.equal(o, want) for o in outs)


@pytest.mark.parametrize("counts,lengths,room", [([1, 1, 1], [100, 3000, 9], 8000), ([80, 1, 7], [100, 3000, 9], 8000)])
def test_captured_graphs_follow_the_lengths(env, counts, lengths, room):
    """Two graphs of the same inputs, replayed in turn while the sequences grow, against the call itself."""
    torch, cafeq = env
    cache = _cache(env, [room] * 3, 2, 64, 64)
    cache.lengths.copy_(torch.tensor(lengths, dtype=torch.int32))
    n = sum(counts)
    q = torch.randn((n, 4, 64), device="cuda:0").bfloat16()
    s = torch.tensor(_starts(counts), dtype=torch.int32, device="cuda:0")
    cafeq.cache_attend(cache, q, s)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(cafeq.cache_attend(cache, q, s, lse=True))
        graphs.append(g)
    for step in range(6):
        q.copy_(torch.randn((n, 4, 64), device="cuda:0"))
        cache.lengths.add_(37)
        graphs[step % 2].replay()
        graphs[1 - step % 2].replay()
        torch.cuda.synchronize()
        want = cafeq.cache_attend(cache, q, s, lse=True)
        for o in outs:
            assert torch.equal(o[0], want[0]) and torch.equal(o[1], want[1])
    _near(env, cache, q, _starts(counts), *outs[0])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("window", [2 ** 30 - 1, 2 ** 30, 2 ** 31 - 1])
def test_the_largest_windows(env, dtype, causal, window):
    torch, cafeq = env
    for counts, lengths in (([1, 2], [300, 1]), ([90, 5], [70, 300])):       # rows before the beginning too
        cache = _cache(env, lengths, 2, 64, 32)
        starts = torch.tensor(_starts(counts), dtype=torch.int32, device="cuda:0")
        q = torch.randn((sum(counts), 4, 64), device="cuda:0").to(torch.float32 if dtype == "f32" else torch.bfloat16)
        want = cafeq.cache_attend(cache, q, starts, causal=causal, lse=True)
        got = cafeq.cache_attend(cache, q, starts, causal=causal, window=window, lse=True)
        _near(env, cache, q, _starts(counts), *got, causal=causal)
        assert torch.equal(torch.isneginf(got[1]), torch.isneginf(want[1]))


def test_far_more_room_than_tokens(env):
    torch, cafeq = env
    lengths = [700, 3, 64, 5000] * 4
    for counts in ([1] * 16, [40] * 16):
        small = _cache(env, [max(n, m) for n, m in zip(lengths, counts)], 2, 64, 64)
        table = torch.full((16, 1 << 16), -1, dtype=torch.int32, device="cuda:0")
        table[:, :small.table.shape[1]] = small.table
        _run(env, counts, lengths, 4, 2, 64, 64, "bf16", cache=small._replace(table=table), window=0)
        _run(env, counts, lengths, 4, 2, 64, 64, "bf16", cache=small._replace(table=table), window=100)


@pytest.mark.parametrize("rep", [128, 300])
def test_one_key_head_for_many(env, rep):
    for dtype in ("bf16", "f32"):
        _run(env, [1, 0, 3], [200, 5, 70], rep, 1, 64, 32, dtype)
        _run(env, [1], [3000], rep, 1, 128, 64, dtype)


def test_a_cache_whose_tensors_are_replaced_or_moved(env):
    torch, cafeq = env
    cache, other = (_cache(env, [300, 200], 2, 64, 64, seed=s) for s in (1, 2))
    q = torch.randn((2, 4, 64), device="cuda:0")
    s = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda:0")
    one, two = cafeq.cache_attend(cache, q, s), cafeq.cache_attend(other, q, s)
    assert not torch.equal(one, two)
    for name in cache._fields:
        setattr(cache, name, getattr(other, name).detach())      # (the same memory, a tensor of its own)
    assert torch.equal(cafeq.cache_attend(cache, q, s), two)
    cache.k.set_(cache.k.clone())
    other.k.zero_()
    assert torch.equal(cafeq.cache_attend(cache, q, s), two)
    cache.k.set_(cache.k[:, :, :, :32])
    with pytest.raises(cafeq.CafeqError):
        cafeq.cache_attend(cache, q, s)
    cache.k = None
    with pytest.raises((cafeq.CafeqError, AttributeError)):
        cafeq.cache_attend(cache, q, s)


def test_refusals(env):
    torch, cafeq = env
    cache = _cache(env, [100, 50], 2, 64, 32)
    q = torch.randn((4, 4, 64), device="cuda:0")
    s = torch.tensor([0, 2, 4], dtype=torch.int32, device="cuda:0")
    for bad in (q.double(), q[:, :3], q[:, :, :32], q.cpu(), q[0], q.transpose(1, 2)):
        with pytest.raises(cafeq.CafeqError):
            cafeq.cache_attend(cache, bad, s)
    for kw in (dict(window=-1), dict(softcap=-1.0), dict(longest=-1), dict(out=q), dict(out=torch.empty_like(q, dtype=torch.bfloat16)), dict(out=torch.empty_like(q)[:3])):
        with pytest.raises(cafeq.CafeqError):
            cafeq.cache_attend(cache, q, s, **kw)
    for starts in (s.long(), s[:2], s.cpu(), s.float()):
        with pytest.raises(cafeq.CafeqError):
            cafeq.cache_attend(cache, q, starts)
    assert cafeq.cache_attend(cache, q[:0], s).shape == (0, 4, 64)
