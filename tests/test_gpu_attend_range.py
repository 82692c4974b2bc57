"""GPU: numbers at the ends of what the attention call takes, and beyond them."""
import pytest

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
