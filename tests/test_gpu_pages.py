"""GPU parity: pages of the cache (cafeq_cache_reserve, cafeq_cache_reorder, cafeq_cache_compact) against the same rules on lists: whole
numbers, equal."""
import numpy as np
import pytest

from tests import cache_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2511_19705_amd import cafeq
    return torch, cafeq


def _pair(env, seqs, pages, heads=2, d=32, block=16, width=6, seed=0):
    """An empty cache whose pages hold random codes, so that copies show."""
    torch, cafeq = env
    rng = np.random.default_rng(seed)
    pool = R.Pool(seqs, pages, heads, d, block, width)
    for side in range(2):
        pool.codes[side][:] = rng.integers(-127, 128, pool.codes[side].shape)
        pool.scales[side][:] = rng.random(pool.scales[side].shape)
    cache = cafeq.kv_cache(seqs, pages, heads, d, block=block, width=width)
    cache.k.copy_(torch.from_numpy(pool.codes[0]))
    cache.v.copy_(torch.from_numpy(pool.codes[1]).transpose(2, 3))
    cache.kscale.copy_(torch.from_numpy(pool.scales[0]))
    cache.vscale.copy_(torch.from_numpy(pool.scales[1]))
    return cache, pool


def _ints(torch, v):
    return torch.tensor([int(x) for x in v], dtype=torch.int32, device="cuda:0")


def _equal(cache, pool):
    for got, want in ((cache.table, pool.table), (cache.lengths, pool.lengths), (cache.refs, pool.refs), (cache.k, pool.codes[0]),
                      (cache.v.transpose(2, 3), pool.codes[1]), (cache.kscale, pool.scales[0]), (cache.vscale, pool.scales[1])):
        assert np.array_equal(got.cpu().numpy(), want)


def _reserve(env, cache, pool, counts):
    torch, cafeq = env
    starts = np.concatenate(([0], np.cumsum(counts)))
    r = cafeq.cache_reserve(cache, _ints(torch, starts), int(starts[-1]))
    want, missing = pool.reserve(list(counts))
    assert int(r.missing) == missing
    if want is not None:
        assert np.array_equal(r.positions.cpu().numpy(), want)
    _equal(cache, pool)
    return missing


def _reorder(env, cache, pool, sources):
    env[1].cache_reorder(cache, _ints(env[0], sources))
    pool.reorder(sources)
    _equal(cache, pool)


def _compact(env, cache, pool):
    assert int(env[1].cache_compact(cache)) == pool.compact()
    _equal(cache, pool)


@pytest.mark.parametrize("block", [16, 32, 64, 128])
def test_a_batch_grows_forks_ends_and_is_compacted(env, block):
    cache, pool = _pair(env, 6, 40, block=block)
    _reserve(env, cache, pool, [block + 3, 1, 0, 2 * block, block - 1, 0])
    _reserve(env, cache, pool, [1] * 6)
    _reorder(env, cache, pool, [0, 1, 0, 3, 0, 1])          # rows 2, 4 and 5 go on from others
    _reserve(env, cache, pool, [1, 1, 1, 0, 1, 1])          # shared pages are copied
    _reserve(env, cache, pool, [block, 0, 1, 1, 0, 2])
    _reorder(env, cache, pool, [5, 4, 3, 2, 1, 0])
    _reorder(env, cache, pool, [-1, 1, 99, 3, -2 ** 31, 5])  # three rows let go
    _reserve(env, cache, pool, [2 * block + 1, 1, 0, 0, 0, 1])
    _compact(env, cache, pool)
    _compact(env, cache, pool)                              # nothing left to move
    _reserve(env, cache, pool, [0, 0, 3, 0, block, 0])
    _reorder(env, cache, pool, [-1] * 6)
    assert (pool.refs == 0).all()
    _compact(env, cache, pool)


def test_no_room_changes_nothing(env):
    cache, pool = _pair(env, 3, 5)
    assert _reserve(env, cache, pool, [40, 0, 1]) == 0      # 4 of 5 pages
    assert _reserve(env, cache, pool, [1, 33, 0]) == 2
    assert _reserve(env, cache, pool, [0, 0, 100]) == 1     # past the table's six columns
    assert _reserve(env, cache, pool, [5, 16, 0]) == 0      # the last one
    assert _reserve(env, cache, pool, [0, 1, 0]) == 1
    _reorder(env, cache, pool, [0, 0, 2])
    assert _reserve(env, cache, pool, [1, 1, 1]) == 1       # copies need room too
    _reorder(env, cache, pool, [0, -1, -1])
    assert _reserve(env, cache, pool, [1, 1, 0]) == 0


@pytest.mark.parametrize("seqs,pages", [(1, 1), (64, 300), (1025, 4200), (3000, 9001)])
def test_many_sequences_and_pages(env, seqs, pages):
    cache, pool = _pair(env, seqs, pages, heads=1, d=16, width=4)
    rng = np.random.default_rng(seqs)
    _reserve(env, cache, pool, rng.integers(0, 30, seqs))
    for _ in range(2):
        _reorder(env, cache, pool, np.where(rng.random(seqs) < 0.3, rng.integers(-1, seqs, seqs), np.arange(seqs)))
        _reserve(env, cache, pool, rng.integers(0, 9, seqs))
        _compact(env, cache, pool)


def test_large_pages_are_copied_whole(env):
    cache, pool = _pair(env, 4, 30, heads=9, d=256, block=128, width=5)
    _reserve(env, cache, pool, [300, 0, 0, 5])
    _reorder(env, cache, pool, [0, 0, 0, -1])
    _reserve(env, cache, pool, [1, 1, 0, 0])
    _reorder(env, cache, pool, [-1, 1, -1, -1])
    _compact(env, cache, pool)


def test_tables_with_numbers_out_of_range(env):
    torch, cafeq = env
    cache, pool = _pair(env, 3, 12)
    _reserve(env, cache, pool, [40, 20, 7])
    for v in (-7, 12, 2 ** 31 - 1):
        cache.table[0, 2] = v
        cafeq.cache_reorder(cache, _ints(torch, [0, 0, 2]))
        cafeq.cache_reserve(cache, _ints(torch, [0, 1, 2, 3]), 3)
        cafeq.cache_compact(cache)
        cafeq.cache_reorder(cache, _ints(torch, [1, -1, -1]))
    torch.cuda.synchronize()


def test_calls_in_a_captured_graph(env):
    torch, cafeq = env
    cache, pool = _pair(env, 4, 60, width=20)
    _reserve(env, cache, pool, [5, 9, 0, 0])
    sources, starts = _ints(torch, [0, 1, 0, 1]), _ints(torch, [0, 1, 3, 7, 7])
    cafeq.cache_reorder(cache._replace(**{n: getattr(cache, n).clone() for n in cache._fields}), sources)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cafeq.cache_reorder(cache, sources)
        r = cafeq.cache_reserve(cache, starts, 7)
        used = cafeq.cache_compact(cache)
    for _ in range(5):
        graph.replay()
        torch.cuda.synchronize()
        pool.reorder([0, 1, 0, 1])
        want, _ = pool.reserve([1, 2, 4, 0])
        assert np.array_equal(r.positions.cpu().numpy(), want) and int(r.missing) == 0
        assert int(used) == pool.compact()
        _equal(cache, pool)


def test_no_sequences(env):
    torch, cafeq = env
    cache = cafeq.kv_cache(0, 3, 1, 16)
    assert int(cafeq.cache_reserve(cache, _ints(torch, [0]), 0).missing) == 0
    cafeq.cache_reorder(cache, _ints(torch, []))
    assert int(cafeq.cache_compact(cache)) == 0
