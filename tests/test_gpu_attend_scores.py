"""GPU parity: attention over the 8-bit cache where scores are far beyond what a softmax of ordinary models meets, against float64 on the same codes.

Scores are float32 numbers: of magnitude s they are known to s 2^-24 and more, so a row's weights follow from its scores only where those are exact or
far enough apart.  Two kinds of inputs:
* exact: one channel of q is not zero (a power of two), scales of k are powers of two.  Scores with equal products code * scale are then the same float32 number, the
  others differ by 2^-8 of the largest and more, which leaves them no weight: out is the mean of V over the largest.  |out - ref| <= r W + h |out| + 2^-36 floor, W the
  mean of |V|; r = 2^-11 for results of bfloat16 (weights to 2^-12, the mantissa of a scale through log2 and exp2, good to 2^-21 each, and where scores stay below
  2^12 the page's exponent less the largest one to 2^-12 ln 2) or 2^-20 (weights in two parts 2^-22, exp2 2^-22, sums), h = 2^-8 or 0.
  Weights p 2^14 mant below 2^-14 are subnormal in float16: each key that has any is off by 2^-25 at most, however small p is, against a denominator above
  2^13 2^-exp of the key with the largest p vs: 2^-38 vs sum |c| over the keys with p > 0, that vs, "floor".  |lse - ref| <= 2^-20 |ref| (eight roundings at
  most) + 2^-10.  Where different scores lie within 64 of the largest one (its magnitude is then below 64 * 2^6), each is off by 8 u of itself, weights and
  their sum by 32 u of it: r grows by that.  Keys on pages of zeros take their rounded score, the others below 2^12 the product itself: u of it, in log2, between them.
* random: with E the bound on a score's error (as in test_gpu_attend: ((2 d + 16) u + 2^-22) sum |q K|), keys more than 2 E + 64 below the largest have no weight
  to speak of (N e^-64), and out lies between the least and the largest V of the others, to r of the largest |V| and h of itself; lse within E + log N of the largest."""
import math

import pytest

from tests.test_gpu_attend import _cache, _starts

pytestmark = pytest.mark.gpu

FORMS = [([1, 1, 1], [900, 64, 300]), ([100, 2, 70], [900, 64, 300])]      # the kernels of few and of many rows


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2511_19705_amd import cafeq
    return torch, cafeq


def _keys(cache, i, h):
    """float64 (K, V, scale of V of each key, |code| of V) of sequence i and key head h."""
    n, B = int(cache.lengths[i]), cache.k.shape[2]
    page = cache.table[i, :-(-n // B)].long()
    K = (cache.k[page, h].double() * cache.kscale[page, h].double()[:, None, None]).reshape(-1, cache.k.shape[3])[:n]
    codes = cache.v[page, h].double().transpose(1, 2).reshape(-1, cache.k.shape[3])[:n]
    vs = cache.vscale[page, h].double().repeat_interleave(B)[:n]
    return K, codes * vs[:, None], vs, codes.abs()


def _rows(cache, q, starts):
    """Every (row, query head, scores' parts): yields (row, g, x, K, V, vs, codes) with the keys in causal reach."""
    hq, heads = q.shape[1], cache.k.shape[1]
    for i in range(len(starts) - 1):
        m, n = starts[i + 1] - starts[i], int(cache.lengths[i])
        for h in range(heads):
            K, V, vs, codes = _keys(cache, i, h)
            for j in range(m):
                end = n - m + j + 1
                for g in range(h * (hq // heads), (h + 1) * (hq // heads)):
                    yield starts[i] + j, g, q[starts[i] + j, g].double(), K[:end], V[:end], vs[:end], codes[:end]


def _exact(env, cache, q, starts, out, lse, scale, cap=0.0, zeros=False):
    torch, f32 = env[0], q.dtype == env[0].float32
    r, h = (2.0 ** -20, 0.0) if f32 else (2.0 ** -11, 2.0 ** -8)
    for row, g, x, K, V, vs, codes in _rows(cache, q, starts):
        s = K @ x * scale
        if cap:
            s = cap * torch.tanh(s / cap)
        top = s.max()
        p = torch.exp(s - top)
        total = p.sum()
        p = p / total
        want, W, floor = p @ V, p @ V.abs(), vs[(p * vs).argmax()] * codes[p > 0].sum(0)
        got = out[row, g].double()
        near = s[s >= top - 64]
        more = 32 * 2.0 ** -24 * float(top.abs()) if float(near.min()) < float(top) else 0.0
        if zeros and abs(float(top)) * 1.4427 < 2.0 ** 12:
            more += 2.0 ** -24 * 1.4427 * abs(float(top))
        tol = (r + more) * W + h * want.abs() + 2.0 ** -36 * floor + 1e-37
        assert torch.isfinite(got).all(), (row, g)
        assert ((got - want).abs() <= tol).all(), (row, g, float(((got - want).abs() / tol).max()))
        ref = float(top + torch.log(total))
        assert abs(float(lse[row, g]) - ref) <= 2.0 ** -20 * abs(ref) + 2.0 ** -10, (row, g, float(lse[row, g]), ref)


def _between(env, cache, q, starts, out, lse, scale):
    torch, f32 = env[0], q.dtype == env[0].float32
    r, h, d = (2.0 ** -20, 0.0, q.shape[2]) if f32 else (2.0 ** -11, 2.0 ** -8, q.shape[2])
    for row, g, x, K, V, _, _ in _rows(cache, q, starts):
        s = K @ x * scale
        E = ((2 * d + 16) * 2.0 ** -24 + 2.0 ** -22) * float((K.abs() @ x.abs()).max()) * abs(scale)
        near = V[s >= s.max() - 2 * E - 64]
        got, slack = out[row, g].double(), r * float(V.abs().max())
        lo, hi = near.min(0).values, near.max(0).values
        assert torch.isfinite(got).all(), (row, g)
        assert (got >= lo - slack - h * lo.abs()).all() and (got <= hi + slack + h * hi.abs()).all(), (row, g)
        assert abs(float(lse[row, g]) - float(s.max())) <= E + math.log(len(V)) + 2.0 ** -20 * abs(float(s.max()))


def _call(env, cache, q, counts, **kw):
    torch, cafeq = env
    s = torch.tensor(_starts(counts), dtype=torch.int32, device="cuda:0")
    return cafeq.cache_attend(cache, q, s, lse=True, **kw)


def _single(env, cache, counts, dtype, exponents, seed=0, hq=4):
    """q with one channel of +-2^e in each row and head; codes of k anew, from a few values so that the largest are met often."""
    torch, _ = env
    gen = torch.Generator(device="cuda:0").manual_seed(seed)
    n, d = sum(counts), cache.k.shape[3]
    cache.k.copy_(torch.randint(-12, 13, cache.k.shape, generator=gen, device="cuda:0") * 10)
    cache.kscale.copy_(2.0 ** torch.randint(-1, 2, cache.kscale.shape, generator=gen, device="cuda:0").float())
    e = torch.tensor(exponents, device="cuda:0")[torch.randint(0, len(exponents), (n, hq), generator=gen, device="cuda:0")].float()
    sign = torch.randint(0, 2, (n, hq), generator=gen, device="cuda:0").float() * 2 - 1
    q = torch.zeros((n, hq, d), device="cuda:0")
    q.scatter_(2, torch.randint(0, d, (n, hq, 1), generator=gen, device="cuda:0"), (sign * 2.0 ** e)[:, :, None])
    return q.to(torch.float32 if dtype == "f32" else torch.bfloat16)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 80, 128, 192, 256])
@pytest.mark.parametrize("exponents", [[17], [20], [24], [27], [31], [40], [70], [110], [8, 14, 17, 20, 24, 29, 34, 90]])
def test_exact_scores(env, dtype, d, exponents):
    for counts, lengths in FORMS:
        cache = _cache(env, lengths, 2, d, 64, seed=d)
        q = _single(env, cache, counts, dtype, exponents, seed=exponents[0] + d)
        _exact(env, cache, q, _starts(counts), *_call(env, cache, q, counts, scale=0.125), 0.125)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("block", [16, 32, 128])
@pytest.mark.parametrize("order", ["up", "down", "mixed", "scales of v", "zeros", "one sign"])
def test_scores_that_grow_from_page_to_page(env, dtype, block, order):
    torch, _ = env
    for counts, lengths in FORMS:
        cache = _cache(env, lengths, 2, 64, block, seed=block)
        q = _single(env, cache, counts, dtype, [2, 20, 40], seed=block)
        for i in range(3):
            page = cache.table[i, :-(-lengths[i] // block)].long()
            step = torch.arange(len(page), device="cuda:0").float()
            power = {"up": step, "down": -step, "mixed": (step * 7) % 11}.get(order, (step * 5) % 3) * (40.0 / max(len(page), 11))
            cache.kscale[page] = (2.0 ** power.round())[:, None].expand(-1, 2).contiguous()
            if order == "scales of v":
                cache.vscale[page] = (2.0 ** ((step * 13) % 61 - 30))[:, None].expand(-1, 2).contiguous()
            if order == "zeros":
                cache.vscale[page[::2]], cache.v[page[::2]] = 0.0, 0
        if order == "one sign":
            cache.k.abs_().clamp_(min=10)
        _exact(env, cache, q, _starts(counts), *_call(env, cache, q, counts, scale=0.125), 0.125, zeros=order == "zeros")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("magnitude", [1e3, 1e4, 1e5, 1e9, 1e17])
def test_random_scores(env, dtype, magnitude):
    """q and what the codes of k stand for of about this magnitude."""
    torch, _ = env
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    for d in (64, 256):
        for counts, lengths in FORMS:
            cache = _cache(env, lengths, 2, d, 64, seed=d)
            cache.kscale.mul_(magnitude)
            q = (torch.randn((sum(counts), 4, d), generator=torch.Generator(device="cuda:0").manual_seed(d), device="cuda:0") * magnitude).to(t)
            for scale in (d ** -0.5, -1.0):
                _between(env, cache, q, _starts(counts), *_call(env, cache, q, counts, scale=scale), scale)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("sign", [-1.0, 1.0])
def test_the_largest_scores_of_float32(env, dtype, sign):
    """All scores of a row +-1.6e38, 2.3e38 in log2: the mean of V, and no row without keys."""
    torch, _ = env
    for counts, lengths in FORMS:
        cache = _cache(env, lengths, 2, 64, 64)
        q = _single(env, cache, counts, dtype, [0])
        cache.k.fill_(120)
        cache.kscale.fill_(2.0 ** 60)
        q = (q.abs() * sign * 2.0 ** 63).to(q.dtype)
        _exact(env, cache, q, _starts(counts), *_call(env, cache, q, counts, scale=0.125), 0.125)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_ordinary_rows_beside_large_ones_keep_their_bits(env, dtype):
    torch, _ = env
    for counts, lengths in FORMS:
        for d in (64, 256):
            cache = _cache(env, lengths, 2, d, 64)
            q = torch.randn((sum(counts), 4, d), device="cuda:0").to(torch.float32 if dtype == "f32" else torch.bfloat16)
            want = _call(env, cache, q, counts)
            large = torch.rand((sum(counts), 4), device="cuda:0") < 0.3
            q2 = torch.where(large[:, :, None], q * 2.0 ** 40, q)
            got = _call(env, cache, q2, counts)
            assert torch.equal(got[0][~large], want[0][~large]) and torch.equal(got[1][~large], want[1][~large])
            assert torch.isfinite(got[0]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,causal", [(50, True), (0, False), (70, False)])
def test_windows_over_large_scores(env, dtype, window, causal):
    """Against the same call on scores that pick the same keys: q times 2^30 and 2^60 give one result."""
    torch, _ = env
    for counts, lengths in FORMS:
        cache = _cache(env, lengths, 2, 64, 32)
        q = _single(env, cache, counts, dtype, [20])
        a = _call(env, cache, (q * 2.0 ** 10).to(q.dtype), counts, scale=0.125, window=window, causal=causal)
        b = _call(env, cache, (q * 2.0 ** 40).to(q.dtype), counts, scale=0.125, window=window, causal=causal)
        assert torch.equal(a[0], b[0]) and torch.isfinite(a[0]).all()
        reach = (torch.ones((), device="cuda:0") * 2.0 ** 30).double()
        assert ((b[1].double() / reach - a[1].double()).abs() <= 2.0 ** -20 * a[1].double().abs() + 16).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_what_is_no_number_beside_large_scores(env, dtype, bad):
    torch, _ = env
    for counts, lengths in FORMS:
        cache = _cache(env, lengths, 2, 64, 64)
        q = _single(env, cache, counts, dtype, [30])
        want = _call(env, cache, q, counts, scale=0.125)
        q2 = q.clone()
        q2[0, 1, 5] = bad
        got = _call(env, cache, q2, counts, scale=0.125)
        assert torch.isnan(got[0][0, 1]).all()
        got[0][0, 1], got[1][0, 1] = want[0][0, 1], want[1][0, 1]
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        # a scale of k or v that is no number, in reach of sequence 0 only
        for side in ("kscale", "vscale"):
            keep = getattr(cache, side).clone()
            getattr(cache, side)[cache.table[0, 2], 0] = bad
            cache.k[cache.table[0, 2], 0], cache.v[cache.table[0, 2], 0] = 0, 0
            got = _call(env, cache, q, counts, scale=0.125)
            assert torch.isnan(got[0][:counts[0], :2]).all()
            assert torch.equal(got[0][:counts[0], 2:], want[0][:counts[0], 2:]) and torch.equal(got[0][counts[0]:], want[0][counts[0]:])
            getattr(cache, side).copy_(keep)
