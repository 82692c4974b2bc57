"""The calls between the projections as they are used together: prompts in chunks, continuations that share pages, single tokens in a captured
graph, rows that end, a pool that is compacted.  Every attention is checked against float64 on what the cache holds (tolerance as derived in
test_gpu_attend), the cache against its recipe bit by bit, pages and positions against lists."""
import importlib.util
import os

import numpy as np
import pytest

from tests import cache_ref as R
from tests.test_gpu_attend import _near
from tests.test_gpu_rotate import _near as _turned

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "serve_attention.py")


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2511_19705_amd import cafeq
    return torch, cafeq


class Run:
    """The library's calls and the reference's, side by side."""

    def __init__(self, env, rows, pages, hq, h, d, block, width, dtype, **attend):
        torch, cafeq = self.env = env
        self.hq, self.h, self.d, self.dtype, self.attend = hq, h, d, dtype, attend
        self.cache = cafeq.kv_cache(rows, pages, h, d, block=block, width=width)
        self.pool = R.Pool(rows, pages, h, d, block, width)
        self.freq, self.amplitude = cafeq.rotary_frequencies(d, scaling="parts", factor=4.0, trained=64, device="cuda:0")
        self.gen = torch.Generator(device="cuda:0").manual_seed(d + rows)
        self.gq, self.gk = (torch.randn(d, generator=self.gen, device="cuda:0") * 0.2 for _ in range(2))

    def ints(self, v):
        return self.env[0].tensor([int(x) for x in v], dtype=self.env[0].int32, device="cuda:0")

    def projected(self, n):
        x = self.env[0].randn((n, (self.hq + 2 * self.h) * self.d), generator=self.gen, device="cuda:0")
        return (x * 2).to(self.dtype)

    def split(self, x):
        at = [0, self.hq, self.hq + self.h, self.hq + 2 * self.h]
        return [x[:, a * self.d:b * self.d].unflatten(1, (b - a, self.d)) for a, b in zip(at, at[1:])]

    def calls(self, x, starts, n, longest):
        _, cafeq = self.env
        q, k, v = self.split(x)
        positions = cafeq.cache_reserve(self.cache, starts, n).positions
        q, k = cafeq.rotate_heads(q, k, positions, self.freq, norm=True, gain_q=self.gq, gain_k=self.gk, gain_offset=1.0, amplitude=self.amplitude)
        cafeq.cache_append(self.cache, k, v, starts, longest=longest)
        return positions, q, k, cafeq.cache_attend(self.cache, q, starts, longest=longest, lse=True, **self.attend)

    def check(self, x, counts, positions, q, k, result):
        torch, _ = self.env
        starts = [0] + list(np.cumsum(counts))
        want, missing = self.pool.reserve(list(counts))
        assert missing == 0 and np.array_equal(positions.cpu().numpy(), want)
        raw = self.split(x)
        for got, y, g in ((q, raw[0], self.gq), (k, raw[1], self.gk)):
            _turned(torch, got, y, positions, self.freq, False, True, g, 1e-6, 1.0, self.amplitude)
        self.pool.append(k.float().cpu().numpy(), raw[2].float().cpu().numpy(), starts)
        self.same()
        _near(self.env, self.cache, q, starts, result[0], result[1], **self.attend)

    def same(self):
        c, p = self.cache, self.pool
        for got, want in ((c.table, p.table), (c.lengths, p.lengths), (c.refs, p.refs)):
            assert np.array_equal(got.cpu().numpy(), want)
        for side, (codes, scales) in enumerate(((c.k, c.kscale), (c.v.transpose(2, 3), c.vscale))):
            live = p.refs > 0
            assert np.array_equal(scales.cpu().numpy()[live], p.scales[side][live])
            codes = codes.cpu().numpy()
            for i, n in enumerate(p.lengths):        # places behind a sequence's tokens hold anything
                for b in range(p.blocks(n)):
                    m = min(p.block, n - b * p.block)
                    assert np.array_equal(codes[p.table[i, b], :, :m], p.codes[side][p.table[i, b], :, :m])

    def step(self, counts):
        x = self.projected(sum(counts))
        self.check(x, counts, *self.calls(x, self.ints([0] + list(np.cumsum(counts))), sum(counts), max(counts)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,h,d,block,attend", [(4, 2, 64, 16, {}), (8, 4, 128, 64, dict(softcap=20.0)), (6, 2, 80, 32, dict(window=70))])
def test_a_served_batch(env, dtype, hq, h, d, block, attend):
    torch, cafeq = env
    run = Run(env, 4, 60, hq, h, d, block, 14, torch.bfloat16 if dtype == "bf16" else torch.float32, **attend)
    run.step([70, 0, 3, 33])            # prompts
    run.step([1, 40, 30, 1])            # a chunk, a new prompt, single tokens
    cafeq.cache_reorder(run.cache, run.ints([0, 0, 2, 0]))
    run.pool.reorder([0, 0, 2, 0])      # rows 1 and 3 go on from row 0
    run.same()
    run.step([1, 1, 1, 1])
    run.step([2, 1, 0, 5])
    # single tokens in a graph
    x, starts = run.projected(4), run.ints(range(5))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        held = run.calls(x, starts, 4, 1)
    for step in range(20):
        x.copy_(run.projected(4))
        graph.replay()
        if step == 10:
            (x + 1).sum().item()        # the program's own work in between
        run.check(x, [1, 1, 1, 1], *held)
    cafeq.cache_reorder(run.cache, run.ints([-1, 1, -1, 3]))
    run.pool.reorder([-1, 1, -1, 3])
    assert int(cafeq.cache_compact(run.cache)) == run.pool.compact()
    run.same()
    graph.replay()
    torch.cuda.synchronize()
    run.check(x, [1, 1, 1, 1], *held)
    run.step([50, 1, 0, 2])


def test_the_layer_is_near_the_one_in_float64(env, capsys):
    """Activations, keys, values and the attention's result in 8 bits, each off by at most 6 / 127 / sqrt(12) = 0.0137 of its standard deviation (a largest
    magnitude of 6 deviations in a group or a page): q, k and v carry the first, k and v their own, the output product another, six in
    all; q, k, v and the two results are rounded to bfloat16 besides.  Scores have a deviation near one, so that their errors pass into the weights as they are."""
    spec = importlib.util.spec_from_file_location("serve_attention", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    for extra, forks in ((["--heads_q", "8", "--heads", "4", "--head", "128"], 2), (["--heads_q", "4", "--heads", "4", "--head", "64", "--softcap", "30"], 3)):
        error, lengths, used = m.main(["--d", "512", "--prompts", "130,77", "--forks", str(forks), "--steps", "5"] + extra)
        assert error < 6 * 0.0137 + 5 * 2.0 ** -8
        assert lengths == [130 + 2 + 5, 77 + 2 + 5] * forks
        # whole blocks of the prompts are shared: 2 of 130 tokens and 1 of 77; behind them each row has its own
        assert used == 2 + 1 + 2 * forks
    assert "us a step" in capsys.readouterr().out
