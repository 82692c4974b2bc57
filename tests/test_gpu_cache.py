"""GPU parity: the 8-bit cache of keys and values (cafeq_cache_append, cafeq_cache_values) against the documented recipe, whose float32
roundings numpy makes too: codes, scales and values are equal bit by bit."""
import numpy as np
import pytest

from tests import cache_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2511_19705_amd import cafeq
    return torch, cafeq


def _pair(env, seqs, pages, heads, d, block, width, seed=0):
    """An empty library cache and its reference, rows of the table over pages in any order."""
    torch, cafeq = env
    pool = R.Pool(seqs, pages, heads, d, block, width)
    order = np.random.default_rng(seed).permutation(pages)[:seqs * width].reshape(seqs, width)
    pool.table[:] = order
    cache = cafeq.kv_cache(seqs, pages, heads, d, block=block, width=width)
    cache.table.copy_(torch.from_numpy(pool.table))
    return cache, pool


def _ints(torch, v):
    return torch.tensor(list(v), dtype=torch.int32, device="cuda:0")


def _equal(torch, cache, pool):
    assert np.array_equal(cache.kscale.cpu().numpy(), pool.scales[0], equal_nan=True)
    assert np.array_equal(cache.vscale.cpu().numpy(), pool.scales[1], equal_nan=True)
    assert np.array_equal(cache.k.cpu().numpy(), pool.codes[0])
    assert np.array_equal(cache.v.transpose(2, 3).cpu().numpy(), pool.codes[1])


def _step(env, cache, pool, counts, dtype, gen, scale=1.0, longest=None, layout="dense", lead=0, tail=0, spoil=None):
    """counts new tokens a sequence into both; rows before and behind the sequences hold numbers that nobody may read."""
    torch, cafeq = env
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    heads, d = cache.k.shape[1], cache.k.shape[3]
    starts = [lead]
    for c in counts:
        starts.append(starts[-1] + c)
    n = starts[-1] + tail
    if layout == "dense":
        k, v = ((torch.randn((n, heads, d), generator=gen, device="cuda:0") * scale).to(t) for _ in range(2))
    elif layout == "fused":
        x = (torch.randn((n, 3 * heads * d), generator=gen, device="cuda:0") * scale).to(t)
        k, v = x[:, heads * d:2 * heads * d].unflatten(1, (heads, d)), x[:, 2 * heads * d:].unflatten(1, (heads, d))
    else:
        k, v = ((torch.randn((heads, n, d), generator=gen, device="cuda:0") * scale).to(t).transpose(0, 1) for _ in range(2))
    if spoil is not None:
        spoil(k, v)
    for x in (k, v):
        x[:lead], x[n - tail:] = float("nan"), float("nan")
    pool.lengths += np.array(counts, np.int32)
    cache.lengths.copy_(torch.from_numpy(pool.lengths))
    cafeq.cache_append(cache, k, v, _ints(torch, starts), longest=longest)
    pool.append(k.float().cpu().numpy(), v.float().cpu().numpy(), starts, longest)
    _equal(torch, cache, pool)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("block", [16, 32, 64, 128])
@pytest.mark.parametrize("heads,d", [(1, 16), (3, 80), (2, 128), (2, 256), (5, 48)])
def test_appending_step_by_step(env, dtype, block, heads, d):
    torch, _ = env
    cache, pool = _pair(env, 4, 64, heads, d, block, 8, seed=d)
    gen = torch.Generator(device="cuda:0").manual_seed(d + block)
    # single tokens, runs that end inside and at the end of a block, several blocks, none; growing and shrinking magnitudes
    for j, counts in enumerate(([1, 0, 3, 16], [1, 2, 13, 0], [2, 30, 0, 1], [block, 1, 2 * block + 1, 1], [0, 0, 0, 0], [1, 1, 1, 1], [3, block - 1, 5, 2])):
        _step(env, cache, pool, counts, dtype, gen, scale=(1.0, 3.0, 0.5, 2.0, 1.0, 9.0, 10.0)[j], lead=j % 2, tail=j % 3)


@pytest.mark.parametrize("layout", ["dense", "fused", "heads first"])
def test_strides(env, layout):
    torch, _ = env
    for dtype in ("f32", "bf16"):
        cache, pool = _pair(env, 2, 20, 3, 64, 32, 8)
        gen = torch.Generator(device="cuda:0").manual_seed(1)
        for counts in ([5, 40], [1, 1], [70, 3]):
            _step(env, cache, pool, counts, dtype, gen, layout=layout)


def test_many_sequences(env):
    torch, _ = env
    gen = torch.Generator(device="cuda:0").manual_seed(2)
    rng = np.random.default_rng(3)
    for seqs in (63, 64, 65, 300, 4100):
        cache, pool = _pair(env, seqs, 3 * seqs, 1, 16, 16, 3)
        for _ in range(2):
            _step(env, cache, pool, list(rng.integers(0, 20, seqs)), "bf16", gen)
        _step(env, cache, pool, [1] * seqs, "bf16", gen, longest=1)
        _step(env, cache, pool, list(rng.integers(0, 2, seqs)), "bf16", gen, longest=1)


def test_rows_beyond_the_bound_are_not_stored(env):
    torch, _ = env
    gen = torch.Generator(device="cuda:0").manual_seed(4)
    for longest in (1, 2, 7, 20):
        cache, pool = _pair(env, 3, 24, 2, 32, 16, 6)
        _step(env, cache, pool, [5, 16, 0], "f32", gen)
        _step(env, cache, pool, [9, 40, 1], "f32", gen, longest=longest)


def test_zeros_tiny_and_huge_numbers(env):
    torch, _ = env
    gen = torch.Generator(device="cuda:0").manual_seed(5)

    def spoil(k, v):
        k[0:8, 0], v[0:8, 1] = 0.0, 0.0
        k[8:16, 0] = 1e-42 * torch.randn((8, 32), generator=gen, device="cuda:0")       # subnormal
        v[8:16, 0] = 3e38
        k[16:24, 1], v[16:24, 1] = 1e-38, -1e30

    cache, pool = _pair(env, 1, 8, 2, 32, 16, 4)
    for counts in ([24], [1], [20]):
        _step(env, cache, pool, counts, "f32", gen, spoil=spoil if counts[0] > 20 else None)
    cache, pool = _pair(env, 1, 8, 2, 32, 16, 4)
    _step(env, cache, pool, [5], "f32", gen, spoil=lambda k, v: (k.zero_(), v.zero_()))
    _step(env, cache, pool, [3], "f32", gen, spoil=lambda k, v: (k.zero_(), v.zero_()))
    _step(env, cache, pool, [3], "f32", gen)
    _step(env, cache, pool, [3], "f32", gen, spoil=lambda k, v: (k.zero_(), v.zero_()))


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_what_is_no_number_stays_in_its_page_and_head(env, bad):
    torch, cafeq = env
    gen = torch.Generator(device="cuda:0").manual_seed(6)

    def spoil(k, v):
        k[2, 0, 3], v[1, 1, 31] = bad, bad

    cache, pool = _pair(env, 2, 16, 3, 32, 16, 4)
    _step(env, cache, pool, [10, 3], "f32", gen)
    _step(env, cache, pool, [4, 3], "bf16", gen, spoil=spoil)
    _step(env, cache, pool, [30, 1], "f32", gen)
    assert (~np.isfinite(pool.scales[0])).sum() == 1 and (~np.isfinite(pool.scales[1])).sum() == 1


def test_pages_that_are_not_there_and_lengths_out_of_range(env):
    torch, cafeq = env
    gen = torch.Generator(device="cuda:0").manual_seed(7)
    cache, pool = _pair(env, 3, 20, 2, 32, 16, 4)
    pool.table[0, 1], pool.table[1, 0], pool.table[2, 2] = -1, 20, 2 ** 31 - 1
    cache.table.copy_(torch.from_numpy(pool.table))
    _step(env, cache, pool, [40, 40, 40], "bf16", gen)
    _step(env, cache, pool, [20, 30, 64], "bf16", gen)      # lengths pass the table's width
    # fewer tokens than rows: the first rows stand before the beginning
    pool.lengths[:] = [3, 0, 20]
    cache.lengths.copy_(torch.from_numpy(pool.lengths))
    starts = [0, 8, 10, 17]
    k, v = (torch.randn((17, 2, 32), generator=gen, device="cuda:0") for _ in range(2))
    cafeq.cache_append(cache, k, v, _ints(torch, starts))
    pool.append(k.cpu().numpy(), v.cpu().numpy(), starts)
    _equal(torch, cache, pool)
    cache.lengths.fill_(-5)
    cafeq.cache_append(cache, k, v, _ints(torch, starts))
    _equal(torch, cache, pool)


@pytest.mark.parametrize("starts", [[5, 3, 9, 2], [-4, 0, 3, 100], [100, 100, 100, 100], [-9, -8, -7, -6], [17, 0, 17, 0]])
def test_rows_out_of_order_write_only_into_pages(env, starts):
    """What such starts mean is open; nothing outside the cache's pages may be written, which guards on both sides show."""
    torch, cafeq = env
    heads, d, B = 2, 32, 16
    cache, _ = _pair(env, 3, 12, heads, d, B, 4)
    size = 12 * heads * B * d
    bufs = [torch.full((size + 8192,), 99, dtype=torch.int8, device="cuda:0") for _ in range(2)]
    cache = cache._replace(k=bufs[0][4096:4096 + size].view(12, heads, B, d), v=bufs[1][4096:4096 + size].view(12, heads, d, B))
    cache.lengths.fill_(40)
    k, v = (torch.randn((17, heads, d), device="cuda:0") for _ in range(2))
    cafeq.cache_append(cache, k, v, _ints(torch, starts))
    cafeq.cache_values(cache, _ints(torch, [0, 3, 30]), _ints(torch, starts), 17)
    cafeq.cache_attend(cache, torch.randn((17, heads, d), device="cuda:0"), _ints(torch, starts))
    torch.cuda.synchronize()
    for b in bufs:
        assert (b[:4096] == 99).all() and (b[4096 + size:] == 99).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("block,heads,d", [(16, 1, 16), (32, 3, 80), (64, 2, 128), (128, 2, 256)])
def test_values(env, dtype, block, heads, d):
    torch, cafeq = env
    gen = torch.Generator(device="cuda:0").manual_seed(8)
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    cache, pool = _pair(env, 4, 40, heads, d, block, 6)
    _step(env, cache, pool, [1, 2 * block, 3 * block + 5, 0], "f32", gen)
    pool.table[2, 1] = -1
    cache.table.copy_(torch.from_numpy(pool.table))
    for begin, counts in (([0, 0, 0, 0], [1, 2 * block, 3 * block + 5, 0]), ([0, 7, block - 1, 0], [0, 3, 2, 4]), ([-3, block, 3 * block, 5], [9, block, 50, 1])):
        starts = [2]
        for c in counts:
            starts.append(starts[-1] + c)
        n = starts[-1] + 1
        got = cafeq.cache_values(cache, _ints(torch, begin), _ints(torch, starts), n, dtype=t)
        for side in range(2):
            assert got[side].shape == (n, heads, d) and got[side].dtype == t
            for i, c in enumerate(counts):
                want = torch.from_numpy(pool.values(side, i, begin[i], c)).to(t)
                assert torch.equal(got[side][starts[i]:starts[i + 1]].cpu(), want)


def test_pages_past_four_gigabytes(env):
    torch, cafeq = env
    heads, d, B = 4, 256, 128
    pages = (1 << 32) // (heads * d * B) + 40
    cache = cafeq.kv_cache(2, 1, heads, d, block=B, width=4)
    cache = cache._replace(k=torch.empty((pages, heads, B, d), dtype=torch.int8, device="cuda:0"), v=torch.empty((pages, heads, d, B), dtype=torch.int8, device="cuda:0"),
                           kscale=torch.zeros((pages, heads), device="cuda:0"), vscale=torch.zeros((pages, heads), device="cuda:0"),
                           refs=torch.zeros(pages, dtype=torch.int32, device="cuda:0"))
    small, pool = _pair(env, 2, 8, heads, d, B, 4)
    far = {p: pages - 1 - int(p) for p in range(8)}
    cache.table.copy_(torch.from_numpy(np.vectorize(far.get)(pool.table).astype(np.int32)))
    gen = torch.Generator(device="cuda:0").manual_seed(9)
    for counts in ([200, 130], [1, 1]):
        n = sum(counts)
        k, v, q = (torch.randn((n, heads, d), generator=gen, device="cuda:0").bfloat16() for _ in range(3))
        starts = _ints(torch, [0, counts[0], n])
        got = []
        pool.lengths += np.array(counts, np.int32)
        for c in (cache, small):
            c.lengths.copy_(torch.from_numpy(pool.lengths))
            cafeq.cache_append(c, k, v, starts)
            got.append(cafeq.cache_values(c, _ints(torch, [0, 0]), _ints(torch, [0] + list(np.cumsum(pool.lengths))), int(pool.lengths.sum()))
                       + (cafeq.cache_attend(c, q, starts),))
        for a, b in zip(*got):
            assert torch.equal(a, b)
    assert torch.equal(cache.k[pages - 8:].flip(0), small.k)


def test_refusals(env):
    torch, cafeq = env
    cache, _ = _pair(env, 2, 8, 2, 32, 16, 4)
    good = torch.randn((4, 2, 32), device="cuda:0")
    starts = _ints(torch, [0, 2, 4])
    odd = torch.randn((4, 2 * 32 + 1), device="cuda:0")[:, :64].unflatten(1, (2, 32))
    for k, v, s in ((good.double(), good.double(), starts), (good, good.bfloat16(), starts), (good[:, :1], good[:, :1], starts), (good, good[:3], starts),
                    (good[:, :, :16], good[:, :, :16], starts), (good, good, starts[:2]), (good, good, starts.long()), (good, good, starts.cpu()), (odd, good, starts),
                    (good.transpose(1, 2), good.transpose(1, 2), starts), (good.cpu(), good.cpu(), starts)):
        with pytest.raises(cafeq.CafeqError):
            cafeq.cache_append(cache, k, v, s)
    for name, t in (("k", cache.k[:, :, :, :16]), ("v", cache.v.transpose(2, 3)), ("kscale", cache.kscale.double()), ("vscale", cache.vscale[:, :1]),
                    ("table", cache.table.long()), ("lengths", cache.lengths[:1]), ("refs", cache.refs.cpu()), ("k", cache.k[0])):
        bad = cache._replace(**{name: t})
        for call in (lambda: cafeq.cache_append(bad, good, good, starts), lambda: cafeq.cache_values(bad, starts[:2], starts, 4),
                     lambda: cafeq.cache_attend(bad, good, starts), lambda: cafeq.cache_reserve(bad, starts, 4), lambda: cafeq.cache_compact(bad)):
            with pytest.raises(cafeq.CafeqError):
                call()
    for kw in (dict(block=8), dict(d=24), dict(d=272), dict(heads=0), dict(pages=0)):
        with pytest.raises(cafeq.CafeqError):
            cafeq.kv_cache(**{**dict(sequences=1, pages=2, heads=1, d=32), **kw})
