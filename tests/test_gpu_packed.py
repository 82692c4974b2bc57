"""GPU parity: products with packed 4-bit weights (cafeq_infer_packed) against float64.

Tolerance, derived from the arithmetic: a code times an activation (or a part of one) is exact in float32.  With 8-bit
activations the sum over a unit of at most 128 columns is an exact integer; a unit's sum then takes three roundings and
the units are added one after another and over at most 16 waves:
    |y - ref| <= 2^-24 (U + 20) sum_units |unit|        U: units of the row
With float activations a unit's products (three parts each) are accumulated in float32, one rounding (counted as 2^-23) each:
    |y - ref| <= 2^-23 (3 * 128 + U + 20) sum_c |q x| s
and, the errors being of either sign, 1e-6 in the 2-norm.  A bfloat16 result adds half a unit in its last place, 2^-9 |y| (2^-8 is used)."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2511_19705_amd import cafeq
    return torch, cafeq


def _weight(rows, cols, group, seed):
    rng = np.random.default_rng(seed)
    codes = rng.integers(-8, 8, (rows, cols)).astype(np.int8)
    scales = np.exp(rng.normal(-4.0, 0.7, (rows, cols // (group or cols)))).astype(np.float32)
    return codes, scales


def _spread(v, group, width):
    return np.repeat(v.astype(np.float64), group or width, axis=1)


def _dev(torch, a):
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda:0")


def _unit(*groups):
    u = 128
    for g, width in groups:
        u = min(u, 128 if g in (0, width) or g % 128 == 0 else 64 if g % 64 == 0 else 32)
    return u


def _check(env, n, rows, cols, group, x_type, xgroup=0, dtype="f32", seed=1, rng_x=None, ld=0):
    torch, cafeq = env
    rng = np.random.default_rng(seed + 77)
    codes, scales = _weight(rows, cols, group, seed)
    W = codes * _spread(scales, group, cols)
    packed = cafeq.pack_nibbles(_dev(torch, codes), _dev(torch, scales), group)
    out_t = torch.float32 if dtype == "f32" else torch.bfloat16
    pad = 0 if not ld else ld - cols
    if x_type == "i8":
        q = rng.integers(-127, 128, (n, cols + pad)).astype(np.int8)
        xs = np.exp(rng.normal(0, 1, (n, cols // (xgroup or cols)))).astype(np.float32)
        x = q[:, :cols] * _spread(xs, xgroup, cols)
        Y = cafeq.infer_packed(_dev(torch, q)[:, :cols], packed, xscales=_dev(torch, xs), xgroup=xgroup, dtype=out_t)
        u = _unit((group, cols), (xgroup, cols))
        edge = range(0, cols, u)
        mag = sum(np.abs(x[:, c:c + u] @ W[:, c:c + u].T) for c in edge)
        bound = 2.0 ** -24 * (len(edge) + 20) * mag
    else:
        x32 = (rng.standard_normal((n, cols + pad)) * np.exp(rng.normal(0, 1.5, (n, 1)))).astype(np.float32)
        xd = _dev(torch, x32)
        if x_type == "bf16":
            xd = xd.to(torch.bfloat16)
        x = xd.double().cpu().numpy()[:, :cols]
        Y = cafeq.infer_packed(xd[:, :cols], packed, dtype=out_t)
        bound = 2.0 ** -23 * (3 * 128 + cols // _unit((group, cols)) + 21) * (np.abs(x) @ np.abs(W).T)
    torch.cuda.synchronize()
    ref = x @ W.T
    got = Y.double().cpu().numpy()
    assert got.shape == (n, rows)
    if dtype == "bf16":
        bound = bound + 2.0 ** -8 * np.abs(ref)
    err = np.abs(got - ref)
    assert np.all(err <= bound), "largest error / bound %.3g" % np.max(err / np.maximum(bound, 1e-300))
    if dtype == "f32":
        assert np.linalg.norm(got - ref) <= 1e-6 * np.linalg.norm(ref)
    return got


@pytest.mark.parametrize("x_type", ["i8", "bf16", "f32"])
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 33, 64, 65, 130, 257])
def test_token_counts(env, n, x_type):
    _check(env, n, 83, 640, 128, x_type, xgroup=128, seed=n)


@pytest.mark.parametrize("x_type", ["i8", "bf16", "f32"])
@pytest.mark.parametrize("rows,cols,group", [(1, 32, 32), (1, 32, 0), (16, 96, 96), (17, 160, 32), (31, 288, 0), (33, 1088, 64),
                                             (129, 2880, 32), (45, 2880, 96), (256, 1152, 384), (300, 4608, 128), (511, 1024, 256)])
@pytest.mark.parametrize("n", [1, 20, 150])
def test_widths_groups_and_ragged_rows(env, rows, cols, group, x_type, n):
    _check(env, n, rows, cols, group, x_type, xgroup=group, seed=rows + cols, dtype="f32")


@pytest.mark.parametrize("group,xgroup", [(128, 0), (128, 64), (64, 128), (32, 256), (0, 32), (256, 128), (96, 576), (0, 0)])
@pytest.mark.parametrize("n", [3, 90])
def test_groups_of_activations_and_weights_need_not_be_the_same(env, group, xgroup, n):
    cols = 1152 if 96 in (group, xgroup) else 1280
    _check(env, n, 70, cols, group, "i8", xgroup=xgroup, seed=group + xgroup)


@pytest.mark.parametrize("x_type", ["i8", "bf16", "f32"])
@pytest.mark.parametrize("n", [1, 40, 300])
def test_results_in_bfloat16_and_strided_activations(env, x_type, n):
    _check(env, n, 200, 1024, 128, x_type, xgroup=128, dtype="bf16", ld=1024 + 48)


@pytest.mark.parametrize("x_type", ["i8", "bf16"])
def test_long_rows_of_one_group(env, x_type):
    _check(env, 2, 40, 36864, 0, x_type, xgroup=0, seed=5)
    _check(env, 2, 17, 65536, 0, x_type, xgroup=0, seed=6)


@pytest.mark.parametrize("n", [1, 5, 70, 200])
def test_extreme_codes_are_exact(env, n):
    # every code -8 or 7, every activation -127 or 127, scales powers of two: all sums are exact
    torch, cafeq = env
    rng = np.random.default_rng(n)
    rows, cols = 48, 4096
    codes = rng.choice(np.array([-8, 7], np.int8), (rows, cols))
    q = rng.choice(np.array([-127, 127], np.int8), (n, cols))
    codes[0], q[0] = -8, 127
    scales = (2.0 ** rng.integers(-3, 3, (rows, cols // 128))).astype(np.float32)
    xs = np.ones((n, 1), np.float32)
    packed = cafeq.pack_nibbles(_dev(torch, codes), _dev(torch, scales), 128)
    Y = cafeq.infer_packed(_dev(torch, q), packed, xscales=_dev(torch, xs), xgroup=0).double().cpu().numpy()
    np.testing.assert_array_equal(Y, (q.astype(np.float64) @ (codes * _spread(scales, 128, cols)).T))


@pytest.mark.parametrize("x_type", ["bf16", "f32"])
@pytest.mark.parametrize("n", [3, 80])
def test_values_that_are_not_finite_stay_in_their_rows(env, x_type, n):
    torch, cafeq = env
    codes, scales = _weight(50, 512, 128, 3)
    codes[codes == 0] = 1                                   # an infinity times zero would be no number
    scales[7, 2] = np.inf
    x = np.random.default_rng(4).standard_normal((n, 512)).astype(np.float32)
    x[1, 100] = np.inf
    x[2, 3] = np.nan
    xd = _dev(torch, x).to(torch.bfloat16 if x_type == "bf16" else torch.float32)
    Y = cafeq.infer_packed(xd, cafeq.pack_nibbles(_dev(torch, codes), _dev(torch, scales), 128)).cpu().numpy()
    bad = np.zeros((n, 50), bool)
    bad[:, 7] = True
    bad[1:3] = True
    np.testing.assert_array_equal(np.isfinite(Y), ~bad)
    keep = np.arange(50) != 7
    np.testing.assert_array_equal(Y[1, keep], np.sign(codes[keep, 100]) * np.float32(np.inf))
    assert np.isnan(Y[2]).all()


@pytest.mark.parametrize("n", [2, 70])
def test_scales_of_activations_that_are_not_finite(env, n):
    torch, cafeq = env
    codes, scales = _weight(33, 256, 64, 3)
    xs = np.ones((n, 4), np.float32)
    xs[0, 1], xs[1, 3] = np.inf, np.nan
    q = np.ones((n, 256), np.int8)
    q[0, 64:128] = 0
    Y = cafeq.infer_packed(_dev(torch, q), cafeq.pack_nibbles(_dev(torch, codes), _dev(torch, scales), 64), xscales=_dev(torch, xs), xgroup=64)
    fin = np.isfinite(Y.cpu().numpy())
    assert not fin[:2].any() and fin[2:].all()


@pytest.mark.parametrize("x_type", ["i8", "f32"])
@pytest.mark.parametrize("n", [4, 100])
def test_output_with_a_stride_touches_nothing_else(env, x_type, n):
    torch, cafeq = env
    codes, scales = _weight(37, 256, 32, 9)
    packed = cafeq.pack_nibbles(_dev(torch, codes), _dev(torch, scales), 32)
    X = torch.ones((n, 256), device="cuda:0", dtype=torch.int8 if x_type == "i8" else torch.float32)
    xs = torch.ones((n, 1), device="cuda:0") if x_type == "i8" else None
    full = torch.full((n + 1, 50), 7.0, device="cuda:0")
    cafeq.infer_packed(X, packed, xscales=xs, out=full[:n, 5:42])
    keep = torch.ones_like(full, dtype=torch.bool)
    keep[:n, 5:42] = False
    assert (full[keep] == 7.0).all()
    ref = (codes * _spread(scales, 32, 256)).sum(1)
    np.testing.assert_allclose(full[:n, 5:42].cpu().numpy(), np.tile(ref, (n, 1)), rtol=0, atol=1e-5 * np.abs(codes * _spread(scales, 32, 256)).sum(1).max())


def test_calls_are_reproducible_and_follow_the_current_stream(env):
    torch, cafeq = env
    codes, scales = _weight(1000, 2304, 128, 12)
    packed = cafeq.pack_nibbles(_dev(torch, codes), _dev(torch, scales), 128)
    for n in (1, 24, 200):
        X = torch.randn((n, 2304), device="cuda:0")
        first = cafeq.infer_packed(X, packed)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            again = [cafeq.infer_packed(X, packed) for _ in range(3)]
        torch.cuda.current_stream().wait_stream(side)
        for y in again:
            assert torch.equal(first, y)


def test_no_tokens(env):
    torch, cafeq = env
    codes, scales = _weight(20, 64, 32, 1)
    Y = cafeq.infer_packed(torch.empty((0, 64), device="cuda:0"), cafeq.pack_nibbles(_dev(torch, codes), _dev(torch, scales), 32))
    assert Y.shape == (0, 20)


def test_agrees_with_the_layer_on_one_byte_codes(env):
    torch, cafeq = env
    g = torch.Generator(device="cuda:0").manual_seed(2)
    W = torch.randn((515, 2304), generator=g, device="cuda:0") * 0.02
    X = torch.randn((6, 2304), generator=g, device="cuda:0")
    for bits in (2, 3, 4):
        codes, scales, _ = cafeq.rtn_quantize(W, bits, 128)
        a = cafeq.infer_single(X, None, codes, scales, 128)
        b = cafeq.infer_packed(X, cafeq.pack_nibbles(codes, scales, 128))
        assert (a - b).norm() <= 2e-6 * a.norm()      # 1e-6 each


def test_refusals(env):
    torch, cafeq = env
    dev = "cuda:0"
    codes, scales = torch.zeros((8, 64), dtype=torch.int8, device=dev), torch.zeros((8, 2), device=dev)
    packed = cafeq.pack_nibbles(codes, scales, 32)
    E = cafeq.CafeqError
    X = torch.zeros((2, 64), device=dev)
    for bad in (lambda: cafeq.pack_nibbles(codes, scales, 64), lambda: cafeq.pack_nibbles(codes, scales, 48),
                lambda: cafeq.pack_nibbles(codes.int(), scales, 32), lambda: cafeq.pack_nibbles(codes[:, :48].contiguous(), scales, 0),
                lambda: cafeq.pack_nibbles(codes.t(), scales, 0), lambda: cafeq.pack_nibbles(codes.cpu(), scales, 32),
                lambda: cafeq.infer_packed(X.double(), packed), lambda: cafeq.infer_packed(X[:, :32], packed),
                lambda: cafeq.infer_packed(X.to(torch.int8), packed), lambda: cafeq.infer_packed(X, packed, xscales=scales),
                lambda: cafeq.infer_packed(X.to(torch.int8), packed, xscales=torch.ones((2, 1), device=dev), xgroup=32),
                lambda: cafeq.infer_packed(X.to(torch.int8), packed, xscales=torch.ones((2, 4), device=dev), xgroup=16),
                lambda: cafeq.infer_packed(X, packed, dtype=torch.float16), lambda: cafeq.infer_packed(X, packed, out=torch.zeros((2, 9), device=dev)),
                lambda: cafeq.infer_packed(torch.zeros((2, 66), device=dev)[:, 1:65], packed), lambda: cafeq.infer_packed(X.cpu(), packed)):
        with pytest.raises(E):
            bad()


def test_activations_and_results_past_two_gigabytes(env):
    # 70000 tokens of 32768 bytes, and as many results of 8192 rows in float32: offsets that no 32 bits hold
    torch, cafeq = env
    rng = np.random.default_rng(8)
    for rows, cols in ((33, 32768), (8192, 256)):
        codes, scales = _weight(rows, cols, 128, 3)
        packed = cafeq.pack_nibbles(_dev(torch, codes), _dev(torch, scales), 128)
        n = 70000
        X = torch.zeros((n, cols), dtype=torch.int8, device="cuda:0")
        at = [0, 1, 65535, 65536, n - 2, n - 1]
        X[at] = _dev(torch, rng.integers(-127, 128, (len(at), cols)).astype(np.int8))
        Y = cafeq.infer_packed(X, packed, xscales=torch.ones((n, 1), device="cuda:0"), xgroup=0)
        ref = X[at].double().cpu().numpy() @ (codes * _spread(scales, 128, cols)).T
        bound = 2.0 ** -24 * (cols // 128 + 20) * sum(np.abs(X[at].double().cpu().numpy()[:, c:c + 128] @ (codes * _spread(scales, 128, cols))[:, c:c + 128].T)
                                                       for c in range(0, cols, 128))
        assert np.all(np.abs(Y[at].double().cpu().numpy() - ref) <= bound)
        rest = torch.ones(n, dtype=torch.bool, device="cuda:0")
        rest[at] = False
        assert not Y[rest].any()
        del X, Y
