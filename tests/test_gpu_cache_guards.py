"""GPU: numbers in device memory that the calls must not trust.  Every buffer that a call writes lies between guards; what the call has no business
with is compared bit by bit."""
import ctypes

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
GUARD = 4096      # bytes on either side


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2511_19705_amd import cafeq
    return torch, cafeq


class Guarded:
    """Tensors in the middle of larger buffers."""

    def __init__(self, torch):
        self.torch, self.buffers = torch, []

    def like(self, t, fill=None):
        torch = self.torch
        size = t.numel() * t.element_size()
        raw = torch.full((size + 2 * GUARD,), 0x5A, dtype=torch.uint8, device="cuda:0")
        inner = raw[GUARD:GUARD + size].view(t.dtype).view(t.shape)
        inner.copy_(t)
        self.buffers.append((raw, size))
        return inner

    def check(self):
        self.torch.cuda.synchronize()
        for raw, size in self.buffers:
            assert (raw[:GUARD] == 0x5A).all() and (raw[GUARD + size:] == 0x5A).all()


def _ints(torch, v):
    return torch.tensor([int(x) for x in v], dtype=torch.int32, device="cuda:0")


def _cache(env, seqs, pages, heads, d, block, width, guarded, seed=0):
    torch, cafeq = env
    gen = torch.Generator(device="cuda:0").manual_seed(seed)
    c = cafeq.kv_cache(seqs, pages, heads, d, block=block, width=width)
    for t in (c.k, c.v):
        t.copy_(torch.randint(-127, 128, t.shape, generator=gen, device="cuda:0"))
    for t in (c.kscale, c.vscale):
        t.copy_(torch.rand(t.shape, generator=gen, device="cuda:0") + 0.1)
    return c._replace(**{n: guarded.like(getattr(c, n)) for n in c._fields})


def _holders(table, lengths, block, pages):
    """How often the rows hold each page of the pool, numbers outside it left out."""
    count = np.zeros(pages, np.int64)
    for row, n in zip(table, lengths):
        for p in row[:-(-max(int(n), 0) // block)]:
            if 0 <= p < pages:
                count[p] += 1
    return count


@pytest.mark.parametrize("width", [8, 4000])      # a table that LDS holds, and one that it does not
@pytest.mark.parametrize("number", [-7, 12, 2 ** 31 - 1, -2 ** 31])
def test_page_numbers_outside_the_pool(env, width, number):
    torch, cafeq = env
    g, B, pages = Guarded(torch), 16, 12
    cache = _cache(env, 5, pages, 2, 32, B, width, g)
    cafeq.cache_reserve(cache, _ints(torch, [0, 40, 60, 67, 67, 67]), 67)      # 3 + 2 + 1 pages
    lost = int(cache.table[0, 2])
    cache.table[0, 2] = number
    cache.refs[lost] = 0                                                        # nobody holds it now
    state = lambda: [t.cpu().numpy().copy() for t in (cache.table, cache.lengths, cache.refs)]      # noqa: E731

    def holds():
        table, lengths, refs = state()
        assert np.array_equal(refs, _holders(table, lengths, B, pages))
        g.check()

    holds()
    codes = [t.clone() for t in (cache.k, cache.v, cache.kscale, cache.vscale)]
    cafeq.cache_reorder(cache, _ints(torch, [0, 0, 2, 0, -5]))                  # the number goes to rows 1 and 3 with the rest of the row
    table, lengths, _ = state()
    assert lengths.tolist() == [40, 40, 7, 40, 0] and (table[:, 2] == [number, number, -1, number, -1]).all()
    holds()
    assert all(torch.equal(a, b) for a, b in zip(codes, (cache.k, cache.v, cache.kscale, cache.vscale)))
    before = state()
    r = cafeq.cache_reserve(cache, _ints(torch, [0, 1, 2, 4, 12, 13]), 13)     # 41, 41, 9, 48 and 1 tokens: one page more for the last row
    assert int(r.missing) == 0
    after = state()
    assert after[1].tolist() == [41, 41, 9, 48, 1] and int((after[0] != before[0]).sum()) == 1
    holds()
    kept = after[2] > 0
    n = np.flatnonzero(kept & (before[2] > 0))
    assert all(torch.equal(a[n], b[n]) for a, b in zip(codes, (cache.k, cache.v, cache.kscale, cache.vscale)))
    used = int(cafeq.cache_compact(cache))
    table, lengths, refs = state()
    assert used == int((refs > 0).sum()) and (refs[:used] > 0).all() and table[0, 2] == number
    holds()
    for row, old in zip(table, after[0]):                                       # moved pages hold what they held
        for p, q in zip(row, old):
            if 0 <= q < pages and before[2][q] > 0:
                assert torch.equal(cache.k[int(p)], codes[0][int(q)]) and torch.equal(cache.vscale[int(p)], codes[3][int(q)])
    cafeq.cache_reorder(cache, _ints(torch, [1, -1, 2 ** 31 - 1, -1, 9]))
    table, lengths, refs = state()
    assert lengths.tolist() == [41, 0, 0, 0, 0]
    holds()


@pytest.mark.parametrize("starts", [[5, 3, 9, 2], [-4, 0, 3, 100], [100, 100, 100, 100], [-9, -8, -7, -6], [17, 0, 17, 0], [0, 17, 2, 17], [2 ** 31 - 1, -2 ** 31, 5, 6],
                                    [17, 17, 17, 0]])
@pytest.mark.parametrize("lengths", [[40, 40, 40], [2 ** 31 - 1, -2 ** 31, 3]])
def test_rows_out_of_order_write_nothing_else(env, starts, lengths):
    """What such rows mean is open; codes, scales, results, sums and values are written, nothing beside them."""
    torch, cafeq = env
    for n, hq in ((17, 2), (17, 34)):
        g, heads, d, B = Guarded(torch), 2, 32, 16
        cache = _cache(env, 3, 12, heads, d, B, 4, g)
        cache.table.copy_(torch.arange(12, device="cuda:0").view(3, 4))
        cache.lengths.copy_(_ints(torch, lengths))
        keep = cache.table.clone(), cache.lengths.clone(), cache.refs.clone()
        s = _ints(torch, starts)
        k, v, q = (torch.randn((n, h, d), device="cuda:0") for h in (heads, heads, hq))
        for longest in (None, 1, 5):
            cafeq.cache_append(cache, k, v, s, longest=longest)
        out, lse = g.like(torch.zeros_like(q)), g.like(torch.zeros((n, hq), device="cuda:0"))
        kv = [g.like(torch.zeros_like(k)) for _ in range(2)]
        c = cafeq._cache(cache, torch.cuda.current_device())[0]
        stream = torch.cuda.current_stream().cuda_stream
        assert cafeq.lib.cafeq_cache_values(ctypes.byref(c), _ints(torch, [0, -30, 2 ** 31 - 1]).data_ptr(), s.data_ptr(), n, kv[0].data_ptr(), kv[1].data_ptr(), 0,
                                            stream) == 0
        for longest in (n, 1):
            a = cafeq.Attention(q.data_ptr(), out.data_ptr(), lse.data_ptr(), n, hq * d, d, hq * d, d, longest, s.data_ptr(), 0, hq, 1, 0, d ** -0.5, 0.0)
            size = cafeq.lib.cafeq_cache_attend_workspace_bytes(ctypes.byref(c), ctypes.byref(a))
            ws = g.like(torch.zeros(max(16, size), dtype=torch.uint8))
            assert cafeq.lib.cafeq_cache_attend(ctypes.byref(c), ctypes.byref(a), ws.data_ptr(), stream) == 0
        g.check()
        assert torch.equal(cache.table, keep[0]) and torch.equal(cache.lengths, keep[1]) and torch.equal(cache.refs, keep[2])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_captured_step_and_an_eager_one_share_nothing(env, dtype):
    """Two graphs over the same cache and inputs, of few and of many rows, and eager calls in between: each has its own scratch."""
    torch, cafeq = env
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    g = Guarded(torch)
    cache = _cache(env, 2, 300, 2, 64, 16, 140, g)
    cafeq.cache_reserve(cache, _ints(torch, [0, 2000, 2100]), 2100)
    jobs = []
    for counts in ([1, 1], [60, 2]):
        n = sum(counts)
        q, s = torch.randn((n, 4, 64), device="cuda:0").to(t), _ints(torch, [0, counts[0], n])
        want = cafeq.cache_attend(cache, q, s, lse=True)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = cafeq.cache_attend(cache, q, s, lse=True)
        jobs.append((graph, got, want, q, s))
    for _ in range(5):
        for graph, got, want, q, s in jobs:
            graph.replay()
            again = cafeq.cache_attend(cache, q, s, lse=True)
            torch.cuda.synchronize()
            for a, b, c in zip(got, want, again):
                assert torch.equal(a, b) and torch.equal(c, b)
    g.check()
