"""GPU: numbers at the ends of what the attention call takes, and beyond them."""
import pytest

from tests import cache_ref as R
from tests.test_gpu_attend import _cache, _starts

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2511_19705_amd import cafeq
    return torch, cafeq


def _problem(env, counts, lengths, dtype="bf16", h=2, d=64):
    torch, _ = env
    gen = torch.Generator(device="cuda:0").manual_seed(d)
    q = torch.randn((sum(counts), 2 * h, d), generator=gen, device="cuda:0").to(torch.float32 if dtype == "f32" else torch.bfloat16)
    return _cache(env, lengths, h, d, 32), q, torch.tensor(_starts(counts), dtype=torch.int32, device="cuda:0")


@pytest.mark.parametrize("counts", [[1, 1], [90, 2]])
def test_integers_that_32_or_64_bits_do_not_hold(env, counts):
    torch, cafeq = env
    cache, q, starts = _problem(env, counts, [300, 200])
    for window in (-1, 1 << 31, (1 << 32) + 100, 1 << 32, -(1 << 32) + 5):
        with pytest.raises(cafeq.CafeqError):
            cafeq.cache_attend(cache, q, starts, window=window)
    want = cafeq.cache_attend(cache, q, starts)
    for longest in (1 << 31, 1 << 63, 1 << 64, (1 << 64) + 1):
        assert torch.equal(cafeq.cache_attend(cache, q, starts, longest=longest), want)
    k = torch.randn((sum(counts), 2, 64), device="cuda:0")
    other = cache._replace(**{n: getattr(cache, n).clone() for n in cache._fields})
    cafeq.cache_append(cache, k, k, starts)
    cafeq.cache_append(other, k, k, starts, longest=1 << 64)
    assert torch.equal(cache.k, other.k) and torch.equal(cache.v, other.v)
    for longest in (-1, -(1 << 64)):
        for call in (lambda: cafeq.cache_attend(cache, q, starts, longest=longest), lambda: cafeq.cache_append(cache, k, k, starts, longest=longest)):
            with pytest.raises(cafeq.CafeqError):
                call()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cap", [200.0, 1e3, 1e4, 1e6, 1e12, 1e30, 3e38, 1e-3, 1e-9, 1e-20, 1e-38, 1e-44])
def test_soft_caps_of_any_size(env, dtype, cap):
    """Scores of a few units and of hundreds under caps far above and below them.  Tolerance for each element as derived in test_gpu_attend; its bound on the
    2-norm besides, 3e-6, is one of scores near one: here each is off by up to 8 u of hundreds, 2^-13, which goes into the weights as it is."""
    torch, _ = env
    for counts, lengths in (([1, 3], [300, 200]), ([90, 2], [300, 200])):
        for d in (64, 256):
            cache, q, starts = _problem(env, counts, lengths, dtype, d=d)
            for scale in (d ** -0.5, 20.0):
                out, lse = env[1].cache_attend(cache, q, starts, softcap=cap, scale=scale, lse=True)
                want, wlse, W, size, floor = R.attend(torch, cache, q, _starts(counts), scale, cap, 0, True)
                u, N, f32 = 2.0 ** -24, 300, dtype == "f32"
                e = 2 * (((2 * d + 16) * u + 2.0 ** -22) * size) + 4 * u
                tol = (2 * e + (2.0 ** -22 if f32 else 2.0 ** -12) + (N + 16) * u)[:, :, None] * W + (0 if f32 else 2.0 ** -8) * want.abs() + 2.0 ** -38 * floor
                assert ((out.double() - want).abs() <= tol + 1e-37).all()
                assert ((lse.double() - wlse).abs() <= 2 * e + (N + 16) * u + 8 * u * wlse.abs()).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_an_infinite_soft_cap_is_none(env, dtype):
    torch, cafeq = env
    for counts in ([1, 3], [90, 2]):
        cache, q, starts = _problem(env, counts, [300, 200], dtype)
        got, want = (cafeq.cache_attend(cache, q, starts, softcap=c, lse=True) for c in (float("inf"), 0.0))
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("power", [-99, -90, -60, 60, 100, 115])
def test_many_keys_of_equal_weight_at_the_ends_of_the_scales(env, dtype, power):
    """Scores of 0 over 70000 keys whose v has scales near 2^power: the mean of V, and the logarithm of their number.  All weights are equal, so that only their sums
    round: a lane adds at most 70000 / 4 of them one after another, waves and parts less than 512 on top, each addition within 2^-24, to the nearest; their errors are
    of either sign, and 2^-14 is 2^10 of them in one direction.  Weights 2^-11 more for bfloat16, as in test_gpu_attend_scores, results 2^-8 of themselves."""
    torch, cafeq = env
    N = 70000
    for n in (1, 100):
        cache, q, starts = _problem(env, [n], [N], dtype)
        cache.vscale.copy_(2.0 ** power * (1 + torch.rand(cache.vscale.shape, device="cuda:0")))
        out, lse = cafeq.cache_attend(cache, q * 0, starts, lse=True)
        keys = torch.arange(N - n + 1, N + 1, device="cuda:0").double()
        assert ((lse.double() - torch.log(keys)[:, None]).abs() <= 2.0 ** -14).all()
        page = cache.table[0, :-(-N // 32)].long()
        for h in range(2):
            V = (cache.v[page, h].double().transpose(1, 2) * cache.vscale[page, h].double()[:, None, None]).reshape(-1, 64)[:N]
            want, W = V.cumsum(0)[N - n:] / keys[:, None], V.abs().cumsum(0)[N - n:] / keys[:, None]
            for g in (2 * h, 2 * h + 1):
                tol = (2.0 ** -14 if dtype == "f32" else 2.0 ** -11 + 2.0 ** -14) * W + (0.0 if dtype == "f32" else 2.0 ** -8) * want.abs()
                assert ((out[:, g].double() - want).abs() <= tol).all()


def test_a_refused_call_leaves_nothing_behind(env):
    """The scratch of a call is known by its sizes; a call of these sizes that is refused needs none, the next one of them does."""
    torch, cafeq = env
    for counts in ([1, 1], [90, 2]):
        cache, q, starts = _problem(env, counts, [3000, 2000])
        apart = torch.zeros((sum(counts), 4 * 64 + 1), device="cuda:0", dtype=q.dtype)[:, :256].unflatten(1, (4, 64))
        for bad in (dict(out=q), dict(softcap=-1.0), dict(out=apart)):
            with pytest.raises(cafeq.CafeqError):
                cafeq.cache_attend(cache, q, starts, **bad)
        want = cafeq.cache_attend(cache, q, starts)
        for i in range(70):      # more sizes than are kept
            cafeq.cache_attend(cache, q, starts, window=1 + i)
        assert torch.equal(cafeq.cache_attend(cache, q, starts), want)
