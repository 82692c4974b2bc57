"""GPU parity: products with packed 4-bit weights in tiles of 32 to 128 tokens (cafeq_infer_packed with many tokens) against float64.

Which way a call goes shows in the workspace that it asks for: float32 activations need three planes of it in tiles and none otherwise (from
17 tokens on the line is the same for all types), and a tile that is split leaves its partial sums there, so many of so many bytes.

Tolerances, from the arithmetic: a code times an activation (or a part of one) is exact in float32.  With 8-bit activations the sum over a unit of at
most 128 columns is an exact integer; it takes at most two roundings on its way to the U units' running sum, up to 20 pieces of the columns are joined
and a token's scale and the result take one each:
    |y - ref| <= 2^-24 (U + 24) sum_units |unit|
With float activations the products of a unit (of each of three parts, P = 3, of float32 ones; P = 1 else) are accumulated one rounding (counted as 2^-23) each:
    |y - ref| <= 2^-23 (128 + P U + 48) sum_c |q x| s
and, the errors being of either sign, 1e-6 in the 2-norm.  A bfloat16 result adds half a unit in its last place, 2^-9 |y| (2^-8 is used)."""
import pytest

pytestmark = pytest.mark.gpu

# (token, row) tiles of 32 of a wave: waves of the workgroup, as the product has them
TILES_I8 = {(1, 1): 4, (2, 1): 4, (2, 2): 4, (4, 2): 8}
TILES_FLOAT = {(1, 1): 4, (2, 1): 4, (2, 2): 8}


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2511_19705_amd import cafeq
    return torch, cafeq


def _kind(cafeq, x_type):
    return {"f32": cafeq.F32, "bf16": cafeq.BF16, "i8": cafeq.I8}[x_type]


def _ways(env, x_type, n, rows, cols, group):
    """(whether the call runs in tiles, the tiles whose split would leave the partial sums that it asks room for)"""
    torch, cafeq = env
    need = lambda t: int(cafeq.lib.cafeq_infer_packed_workspace_bytes(_kind(cafeq, t), n, rows, cols, group))  # noqa: E731
    assert n > 16
    part = need(x_type)
    if x_type == "f32":
        part -= -(-n * cols * 6 // 256) * 256 if part else 0
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    fits = set()
    for (mt, nt), waves in (TILES_I8 if x_type == "i8" else TILES_FLOAT).items():
        tiles = -(-n // (32 * mt)) * -(-rows // (32 * nt * waves))
        rest = tiles % (8 // waves * cus)
        size = 32 * mt * 32 * nt * waves * 4
        if part and rest and part % (rest * size) == 0 and 2 <= part // (rest * size) <= 40:
            fits.add((mt, nt))
    return need("f32") > 0, fits


def _unit(*groups):
    u = 128
    for g, width in groups:
        u = min(u, 128 if g in (0, width) or g % 128 == 0 else 64 if g % 64 == 0 else 32)
    return u


def _weight(torch, rows, cols, group, gen):
    codes = torch.randint(-8, 8, (rows, cols), generator=gen, device="cuda:0", dtype=torch.int8)
    scales = torch.exp(torch.randn((rows, cols // (group or cols)), generator=gen, device="cuda:0") * 0.7 - 4.0)
    return codes, scales


def _activations(torch, n, cols, x_type, xgroup, gen, pad=0):
    """(x as it is given, its scales, its values in float64)"""
    if x_type == "i8":
        x = torch.randint(-127, 128, (n, cols + pad), generator=gen, device="cuda:0", dtype=torch.int8)[:, :cols]
        xs = torch.exp(torch.randn((n, cols // (xgroup or cols)), generator=gen, device="cuda:0"))
        return x, xs, x.double() * xs.double().repeat_interleave(xgroup or cols, 1)
    x = torch.randn((n, cols + pad), generator=gen, device="cuda:0") * torch.exp(torch.randn((n, 1), generator=gen, device="cuda:0") * 1.5)
    x = (x.bfloat16() if x_type == "bf16" else x)[:, :cols]
    return x, None, x.double()


def _bound(torch, x, W, x_type, unit):
    cols = x.shape[1]
    u = -(-cols // unit)
    if x_type != "i8":
        return 2.0 ** -23 * (128 + (3 if x_type == "f32" else 1) * u + 48) * (x.abs() @ W.abs().t().contiguous())
    mag = torch.zeros((x.shape[0], W.shape[0]), dtype=torch.float64, device="cuda:0")
    for c in range(0, cols, unit):
        mag += (x[:, c:c + unit].contiguous() @ W[:, c:c + unit].t().contiguous()).abs()
    return 2.0 ** -24 * (u + 24) * mag


def _check(env, x_type, n, rows, cols, group, xgroup=0, dtype="f32", pad=0, ypad=0, seed=1):
    torch, cafeq = env
    gen = torch.Generator(device="cuda:0").manual_seed(seed + n + 3 * rows + 7 * cols)
    codes, scales = _weight(torch, rows, cols, group, gen)
    x, xs, xv = _activations(torch, n, cols, x_type, xgroup, gen, pad)
    W = codes.double() * scales.double().repeat_interleave(group or cols, 1)
    out_t = torch.float32 if dtype == "f32" else torch.bfloat16
    whole = torch.full((n, rows + ypad), 7.0, device="cuda:0", dtype=out_t)
    got = cafeq.infer_packed(x, cafeq.pack_nibbles(codes, scales, group), xscales=xs, xgroup=xgroup, out=whole[:, :rows])
    ref = xv @ W.t().contiguous()
    bound = _bound(torch, xv, W, x_type, _unit((group, cols), (xgroup, cols)) if x_type == "i8" else _unit((group, cols)))
    if dtype == "bf16":
        bound += 2.0 ** -8 * ref.abs()
    err = (got.double() - ref).abs()
    assert bool((err <= bound).all()), "largest error / bound %.3g" % float((err / bound.clamp(min=1e-300)).max())
    if dtype == "f32":
        assert float((got.double() - ref).norm()) <= 1e-6 * float(ref.norm())
    assert bool((whole[:, rows:] == 7.0).all())
    return got


# units of 32 and 64 columns and of 128 (of one group a row where the width is not a multiple of 128: the last stage is part full)
WIDTHS = {("short", 32): (1184, 32), ("short", 64): (1216, 64), ("short", 128): (1152, 128), ("short", "row"): (1184, 0),
          ("long", 32): (4640, 32), ("long", 64): (4672, 64), ("long", 128): (4608, 128), ("long", "row"): (4640, 0),
          ("longer", 32): (9248, 32), ("longer", 64): (9280, 64), ("longer", 128): (9216, 128), ("longer", "row"): (9248, 0),
          ("middle", 32): (2848, 32), ("middle", 64): (2880, 64), ("middle", 128): (2816, 128), ("middle", "row"): (2848, 0)}
UNITS = [32, 64, 128, "row"]
# every tile with its columns split over workgroups
SPLIT = [("i8", (1, 1), 65, 3500, "long"), ("i8", (2, 1), 700, 300, "long"), ("i8", (2, 2), 700, 2000, "longer"), ("i8", (4, 2), 5003, 3500, "middle"),
         ("bf16", (1, 1), 65, 3500, "long"), ("bf16", (2, 1), 700, 300, "long"), ("bf16", (2, 2), 700, 3500, "long"),
         ("f32", (1, 1), 65, 3500, "long"), ("f32", (2, 1), 700, 300, "long"), ("f32", (2, 2), 65, 9001, "long")]


@pytest.mark.parametrize("unit", UNITS)
@pytest.mark.parametrize("x_type,tile,n,rows,width", SPLIT)
def test_every_tile_split(env, x_type, tile, n, rows, width, unit):
    cols, group = WIDTHS[width, unit]
    tiles, fits = _ways(env, x_type, n, rows, cols, group)
    assert tiles and tile in fits, fits
    _check(env, x_type, n, rows, cols, group)


@pytest.mark.parametrize("unit", [32, 64, 128])
@pytest.mark.parametrize("tile,n,rows,width", [c[1:] for c in SPLIT if c[0] == "i8"])
def test_every_tile_split_with_a_scale_per_group_of_activations(env, tile, n, rows, width, unit):
    cols, group = WIDTHS[width, unit]
    tiles, fits = _ways(env, "i8", n, rows, cols, group)
    assert tiles and tile in fits, fits
    _check(env, "i8", n, rows, cols, group, xgroup=group)


# tiles that one workgroup takes whole, one round of them and more, with a rest that is split and without
@pytest.mark.parametrize("x_type", ["i8", "bf16", "f32"])
@pytest.mark.parametrize("unit", UNITS)
@pytest.mark.parametrize("n,rows", [(700, 1147), (65, 13001), (500, 9001), (300, 7001), (4100, 1000), (4100, 2000)])
def test_whole_tiles(env, n, rows, unit, x_type):
    cols, group = WIDTHS["short", unit]
    assert _ways(env, x_type, n, rows, cols, group)[0]
    _check(env, x_type, n, rows, cols, group, xgroup=group if unit != "row" and n < 1000 else 0)


@pytest.mark.parametrize("unit", UNITS)
def test_whole_tiles_of_128_tokens(env, unit):
    cols, group = WIDTHS["short", unit]
    assert _ways(env, "i8", 3001, 3500, cols, group)[0]
    _check(env, "i8", 3001, 3500, cols, group, xgroup=group)


@pytest.mark.parametrize("group,xgroup", [(128, 0), (128, 64), (64, 128), (32, 256), (0, 32), (256, 128), (96, 576), (576, 96), (0, 0), (384, 0)])
@pytest.mark.parametrize("n,rows", [(700, 1147), (700, 300)])
def test_groups_of_activations_and_weights_need_not_be_the_same(env, group, xgroup, n, rows):
    cols = {(700, 1147): 1152, (700, 300): 4608}[n, rows] if 256 not in (group, xgroup) else {(700, 1147): 1280, (700, 300): 4608}[n, rows]
    assert _ways(env, "i8", n, rows, cols, group)[0]
    _check(env, "i8", n, rows, cols, group, xgroup=xgroup)


@pytest.mark.parametrize("x_type", ["i8", "bf16", "f32"])
@pytest.mark.parametrize("n,rows,width", [(700, 1147, "short"), (700, 300, "long"), (65, 9001, "middle")])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strides_and_results_in_bfloat16(env, n, rows, width, x_type, dtype):
    for unit in (32, 128):
        cols, group = WIDTHS[width, unit]
        assert _ways(env, x_type, n, rows, cols, group)[0]
        _check(env, x_type, n, rows, cols, group, dtype=dtype, pad=48, ypad=13)


# around the line between few tokens and many, and token counts about the tiles' edges
@pytest.mark.parametrize("x_type", ["i8", "bf16", "f32"])
@pytest.mark.parametrize("n", [9, 16, 17, 31, 32, 33, 63, 64, 65, 96, 127, 128, 129])
def test_token_counts(env, n, x_type):
    _check(env, x_type, n, 20011, 2880, 32, xgroup=32)
    _check(env, x_type, n, 20000, 5120, 128, xgroup=128)


# few tokens of a matrix so tall that a wave takes two of its row tiles (8 bits, from three tokens on)
@pytest.mark.parametrize("unit", UNITS)
@pytest.mark.parametrize("n,rows,cols", [(3, 16400, 1184), (8, 16400, 1184), (16, 20011, 2848), (20, 16400, 1184), (32, 17001, 1184), (40, 16400, 1184)])
def test_few_tokens_of_tall_matrices(env, n, rows, cols, unit):
    torch, cafeq = env
    cols += {32: 0, 64: 32, 128: 96, "row": 0}[unit]
    assert cafeq.lib.cafeq_infer_packed_workspace_bytes(cafeq.F32, n, rows, cols, 32) == 0 or n <= 16
    for xgroup in (0, 32 if unit == "row" else unit):
        _check(env, "i8", n, rows, cols, 0 if unit == "row" else unit, xgroup=xgroup)


@pytest.mark.parametrize("n,rows,cols", [(700, 1147, 1184), (700, 300, 4640), (300, 1147, 2880)])
def test_extreme_codes_are_exact(env, n, rows, cols):
    # every code -8 or 7, every activation -127 or 127, scales powers of two: sums below 2^24 units, all exact
    torch, cafeq = env
    assert _ways(env, "i8", n, rows, cols, 32)[0]
    gen = torch.Generator(device="cuda:0").manual_seed(n)
    codes = torch.randint(0, 2, (rows, cols), generator=gen, device="cuda:0", dtype=torch.int8) * 15 - 8
    q = torch.randint(0, 2, (n, cols), generator=gen, device="cuda:0", dtype=torch.int8) * 127
    q = torch.where(q == 0, -127, q).to(torch.int8)
    codes[0], q[0] = -8, 127
    scales = torch.full((rows, cols // 32), 0.25, device="cuda:0")
    Y = cafeq.infer_packed(q, cafeq.pack_nibbles(codes, scales, 32), xscales=torch.ones((n, 1), device="cuda:0"))
    assert torch.equal(Y.double(), q.double() @ (codes.double() * 0.25).t().contiguous())


@pytest.mark.parametrize("x_type", ["i8", "bf16", "f32"])
@pytest.mark.parametrize("n,rows,width", [(700, 1147, "short"), (700, 300, "long"), (65, 9001, "long")])
def test_calls_are_reproducible_on_two_streams_at_once(env, x_type, n, rows, width):
    torch, cafeq = env
    cols, group = WIDTHS[width, 128]
    gen = torch.Generator(device="cuda:0").manual_seed(4)
    packed = cafeq.pack_nibbles(*_weight(torch, rows, cols, group, gen), group)
    calls = [_activations(torch, n, cols, x_type, 0, gen)[:2] for _ in range(2)]
    want = [cafeq.infer_packed(x, packed, xscales=xs) for x, xs in calls]
    streams = [torch.cuda.Stream() for _ in calls]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(4):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[i].append(cafeq.infer_packed(calls[i][0], packed, xscales=calls[i][1]))
    torch.cuda.synchronize()
    for i in range(2):
        for y in got[i]:
            assert torch.equal(y, want[i])


@pytest.mark.parametrize("x_type", ["bf16", "f32"])
def test_a_captured_graph_of_many_tokens_replays(env, x_type):
    torch, cafeq = env
    n, rows, (cols, group) = 700, 300, WIDTHS["long", 32]
    gen = torch.Generator(device="cuda:0").manual_seed(6)
    packed = cafeq.pack_nibbles(*_weight(torch, rows, cols, group, gen), group)
    x, _, _ = _activations(torch, n, cols, x_type, 0, gen)
    assert cafeq.lib.cafeq_infer_packed_workspace_bytes(_kind(cafeq, x_type), n, rows, cols, group) > 0
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        cafeq.infer_packed(x, packed)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = cafeq.infer_packed(x, packed)
    for _ in range(4):
        x.copy_(torch.randn((n, cols), generator=gen, device="cuda:0"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(held, cafeq.infer_packed(x, packed))
