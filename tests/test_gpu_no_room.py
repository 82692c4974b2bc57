"""GPU: a step that finds no room (cafeq_cache_reserve with too few pages or columns) leaves the cache as it is, whatever calls follow it in the
step, eager or in a captured graph: codes, scales, lengths, tables and holders are equal bit by bit."""
import ctypes

import numpy as np
import pytest

from tests import cache_ref as R
from tests.test_gpu_attend import _near

pytestmark = pytest.mark.gpu
HQ, H, D, B = 4, 2, 64, 16


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2511_19705_amd import cafeq
    return torch, cafeq


def _ints(torch, v):
    return torch.tensor([int(x) for x in v], dtype=torch.int32, device="cuda:0")


def _step(env, cache, x, starts, n, longest):
    cafeq = env[1]
    q, k, v = x[:, :HQ], x[:, HQ:HQ + H], x[:, HQ + H:]
    r = cafeq.cache_reserve(cache, starts, n)
    freq, _ = cafeq.rotary_frequencies(D, device="cuda:0")
    q, k = cafeq.rotate_heads(q, k, r.positions, freq)
    cafeq.cache_append(cache, k, v, starts, longest=longest)
    return r, q, k, cafeq.cache_attend(cache, q, starts, longest=longest, lse=True)


def _x(env, n, dtype, seed=0):
    torch = env[0]
    gen = torch.Generator(device="cuda:0").manual_seed(seed)
    return torch.randn((n, HQ + 2 * H, D), generator=gen, device="cuda:0").to(dtype)


def _state(cache):
    return [getattr(cache, n).clone() for n in cache._fields if n != "missing"]


def _same(torch, cache, state):
    return all(torch.equal(getattr(cache, n), t) for n, t in zip((f for f in cache._fields if f != "missing"), state))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("counts", [[1, 1, 0], [40, 3, 0], [100, 0, 0]])
def test_a_step_without_room_leaves_the_cache(env, dtype, counts):
    torch, cafeq = env
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    cache = cafeq.kv_cache(3, 4, H, D, block=B, width=6)
    r, _, _, (out, _) = _step(env, cache, _x(env, 57, t), _ints(torch, [0, 57, 57, 57]), 57, 57)      # all four pages
    assert int(r.missing) == 0 and int(cache.missing) == 0 and bool((out != 0).any())
    cafeq.cache_reorder(cache, _ints(torch, [0, 0, 0]))      # three rows share the last, partly filled page
    span = _ints(torch, [0, 0, 0]), _ints(torch, [0, 57, 57, 57]), 57
    state, held = _state(cache), cafeq.cache_values(cache, *span)
    starts, n = np.concatenate(([0], np.cumsum(counts))), sum(counts)
    for _ in range(2):
        r, _, _, (out, lse) = _step(env, cache, _x(env, n, t, 1), _ints(torch, starts), n, max(counts))
        assert int(r.missing) > 0 and int(cache.missing) == int(r.missing)
        assert _same(torch, cache, state)
        assert (r.positions == 0).all() and (out == 0).all() and torch.isneginf(lse).all()
    # what was stored can be read back; a reserve that finds room opens the cache again
    for a, b in zip(held, cafeq.cache_values(cache, *span)):
        assert torch.equal(a, b)
    cafeq.cache_reorder(cache, _ints(torch, [0, -1, -1]))
    r, q, _, (out, lse) = _step(env, cache, _x(env, 2, t, 2), _ints(torch, [0, 2, 2, 2]), 2, 2)
    assert int(r.missing) == 0 and int(cache.missing) == 0 and r.positions.tolist() == [57, 58]
    _near(env, cache, q, [0, 2, 2, 2], out, lse)


def test_a_captured_step_that_runs_out_of_room(env):
    torch, cafeq = env
    cache = cafeq.kv_cache(2, 5, H, D, block=B, width=8)
    x, starts = _x(env, 2, torch.bfloat16), _ints(torch, [0, 1, 2])
    scratch = cache._replace(**{n: getattr(cache, n).clone() for n in cache._fields})
    _step(env, scratch, x, starts, 2, 1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r, q, k, (out, lse) = _step(env, cache, x, starts, 2, 1)
    pool = R.Pool(2, 5, H, D, B, 8)
    for step in range(40):      # 2 rows grow to 32 tokens each on 4 pages; the 33rd step asks for two and finds one
        x.copy_(_x(env, 2, torch.bfloat16, step))
        graph.replay()
        torch.cuda.synchronize()
        want, missing = pool.reserve([1, 1])
        assert int(r.missing) == missing == (0 if step < 32 else 1)
        if missing == 0:
            pool.append(k.float().cpu().numpy(), x[:, HQ + H:].float().cpu().numpy(), [0, 1, 2])
            assert np.array_equal(r.positions.cpu().numpy(), want)
            _near(env, cache, q, [0, 1, 2], out, lse)
        else:
            assert (out == 0).all() and torch.isneginf(lse).all()
        assert cache.lengths.tolist() == pool.lengths.tolist()
        live = pool.refs > 0
        assert np.array_equal(cache.kscale.cpu().numpy()[live], pool.scales[0][live]) and np.array_equal(cache.vscale.cpu().numpy()[live], pool.scales[1][live])
        assert np.array_equal(cache.k.cpu().numpy()[live], pool.codes[0][live]) and np.array_equal(cache.v.transpose(2, 3).cpu().numpy()[live], pool.codes[1][live])
    cafeq.cache_reorder(cache, _ints(torch, [0, -1]))
    pool.reorder([0, -1])
    graph.replay()
    torch.cuda.synchronize()
    assert int(r.missing) == 0 and r.positions.tolist() == [32, 0] == pool.reserve([1, 1])[0].tolist()


def test_without_a_place_for_it(env):
    """A descriptor whose `missing` is NULL: lengths are the caller's to keep."""
    torch, cafeq = env
    cache = cafeq.kv_cache(1, 2, H, D, block=B)
    x = _x(env, 20, torch.float32)
    _step(env, cache, x, _ints(torch, [0, 20]), 20, 20)
    desc = cafeq.Cache(cache.k.data_ptr(), cache.v.data_ptr(), cache.kscale.data_ptr(), cache.vscale.data_ptr(), cache.table.data_ptr(), cache.lengths.data_ptr(),
                       cache.refs.data_ptr(), 2, 1, 2, H, D, B, None)
    q, out, s = torch.randn((1, HQ, D), device="cuda:0"), torch.empty((1, HQ, D), device="cuda:0"), _ints(torch, [0, 1])
    want = cafeq.cache_attend(cache, q, s)
    cache.missing.fill_(3)
    assert (cafeq.cache_attend(cache, q, s) == 0).all()
    a = cafeq.Attention(q.data_ptr(), out.data_ptr(), None, 1, HQ * D, D, HQ * D, D, 1, s.data_ptr(), 0, HQ, 1, 0, D ** -0.5, 0.0)
    ws = torch.empty(max(16, cafeq.lib.cafeq_cache_attend_workspace_bytes(ctypes.byref(desc), ctypes.byref(a))), dtype=torch.uint8, device="cuda:0")
    assert cafeq.lib.cafeq_cache_attend(ctypes.byref(desc), ctypes.byref(a), ws.data_ptr(), torch.cuda.current_stream().cuda_stream) == 0
    assert torch.equal(out, want)


def test_a_reserve_for_no_token_opens_the_cache(env):
    torch, cafeq = env
    cache = cafeq.kv_cache(1, 2, H, D, block=B)
    _step(env, cache, _x(env, 30, torch.float32), _ints(torch, [0, 30]), 30, 30)
    q, s = torch.randn((1, HQ, D), device="cuda:0"), _ints(torch, [0, 1])
    want = cafeq.cache_attend(cache, q, s)
    assert int(cafeq.cache_reserve(cache, _ints(torch, [0, 9]), 9).missing) == 1
    assert (cafeq.cache_attend(cache, q, s) == 0).all()
    assert int(cafeq.cache_reserve(cache, _ints(torch, [0, 0]), 0).missing) == 0
    assert torch.equal(cafeq.cache_attend(cache, q, s), want) and cache.lengths.tolist() == [30]
