"""GPU parity: activations in 8 bits (cafeq_norm_quantize) against float64.

Tolerances, from the arithmetic in float32 (u = 2^-24): the sum of squares of a row has chains of at most 64 terms and a
tree of at most 16 + 6 levels, half of whose relative error goes to 1 / rms; three products follow:
    |y - ref| <= 64 u |ref|
The transform multiplies parts whose omitted products are below 2^-22 and accumulates 6 k of them:
    |z - ref| <= 2^-23 (6 k + 64) sum_j |Tinv_ij| |y_j|, 2e-6 in the 2-norm
A scale is the largest magnitude of its group over 127, off by as much as the largest error in the group; a code times its scale is
within half a step of z, and the errors of z and of the reciprocal step (127 steps, 4 u each) more:
    |q s - ref| <= s (1/2 + 127 * 4 u) + error of z"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2511_19705_amd import cafeq
    return torch, cafeq


def _reference(x, res, gain, offset, eps, norm, P):
    """h, z and the bound on the error of z, all float64."""
    h = x if res is None else x + res
    y = h.copy()
    if norm:
        y = h / np.sqrt((h * h).mean(1, keepdims=True) + eps)
        if gain is not None:
            y = y * (offset + gain)
    err = 64 * U * np.abs(y) + 1e-44
    if P is None:
        return h, y, err
    nb, k, _ = P.shape
    yb = y.reshape(len(y), nb, k)
    z = np.matmul(yb.transpose(1, 0, 2), P.transpose(0, 2, 1)).transpose(1, 0, 2).reshape(y.shape)
    mag = np.matmul(np.abs(yb).transpose(1, 0, 2), np.abs(P).transpose(0, 2, 1)).transpose(1, 0, 2).reshape(y.shape)
    return h, z, 2 * U * (6 * k + 64) * mag + 1e-44


def _check(env, n, d, dtype="f32", residual=True, gain=True, offset=1.0, norm=True, k=0, group=0, values="f32", pad=0, eps=1e-6,
           seed=0, edit=None):
    torch, cafeq = env
    T = {"f32": torch.float32, "bf16": torch.bfloat16, None: None}
    g = torch.Generator(device="cpu").manual_seed(seed + 13 * d + n)
    x = (torch.randn((n, d + pad), generator=g) * torch.exp(torch.randn((n, 1), generator=g))).to(T[dtype])
    r = torch.randn((n, d + pad), generator=g).to(T[dtype]) if residual else None
    if edit:
        edit(x, r)
    w = torch.randn(d, generator=g) * 0.3 if gain else None
    P = None
    if k:
        P = torch.linalg.qr(torch.randn((d // k, k, k), generator=g))[0] + torch.randn((d // k, k, k), generator=g) * (0.1 / k ** 0.5)
    xd, rd = x.cuda()[:, :d], None if r is None else r.cuda()[:, :d]
    o = cafeq.norm_quantize(xd, None if w is None else w.cuda(), residual=rd, eps=eps, gain_offset=offset, norm=norm,
                            Tinv=None if P is None else P.contiguous().cuda(), group=group, values=T[values])
    torch.cuda.synchronize()
    f64 = lambda t: None if t is None else t.double().numpy()  # noqa: E731
    h, z, err = _reference(f64(x[:, :d]), f64(r[:, :d]) if residual else None, f64(w), offset, eps, norm, f64(P))
    if residual:
        assert torch.equal(o.sum.cpu(), (x[:, :d].float() + r[:, :d].float()).to(T[dtype]))
    else:
        assert o.sum is None
    if group is None:
        assert o.codes is None and o.scales is None
        got = o.values.double().cpu().numpy()
        bound = err if values == "f32" else err + 2.0 ** -8 * np.abs(z)
        assert np.all(np.abs(got - z) <= bound), np.max(np.abs(got - z) / bound)
        if values == "f32" and k:
            assert np.linalg.norm(got - z) <= 2e-6 * np.linalg.norm(z)
        return o
    gl = group or d
    a = np.abs(z).reshape(n, -1, gl).max(2)
    ea = err.reshape(n, -1, gl).max(2)
    s = o.scales.double().cpu().numpy()
    q = o.codes.cpu().numpy()
    assert np.all(np.abs(s - a / 127) <= (ea + 4 * U * a) / 127 + 1e-44)
    assert q.min() >= -127 and q.max() <= 127
    v = q.astype(np.float32) * np.repeat(o.scales.cpu().numpy(), gl, axis=1)
    step = np.repeat(s, gl, axis=1)
    assert np.all(np.abs(v.astype(np.float64) - z) <= step * (0.5 + 127 * 4 * U) + err + 1e-40)
    full = np.abs(q.reshape(n, -1, gl).astype(np.int32)).max(2)
    assert np.all(full[a > 1e-36] == 127)
    if values:
        assert torch.equal(o.values.cpu(), torch.from_numpy(v).to(T[values]))
    else:
        assert o.values is None
    return o


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [1, 2, 5, 8, 31, 33, 64, 255, 1000, 2304, 3584, 4609, 8200, 14336, 20000, 36864, 65536])
def test_row_lengths_with_one_scale(env, d, dtype):
    _check(env, 3, d, dtype, group=0)


@pytest.mark.parametrize("d,group", [(32, 32), (96, 32), (96, 96), (288, 32), (1152, 384), (1024, 512), (2048, 1024), (2880, 32), (2880, 64),
                                     (2880, 576), (4608, 128), (4608, 256), (14336, 128), (36864, 128), (36864, 1536), (65536, 32)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_groups(env, d, group, dtype):
    _check(env, 2, d, dtype, group=group, values="bf16")


@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 100, 700])
def test_token_counts(env, n):
    _check(env, n, 1152, "bf16", group=128)
    _check(env, n, 1152, "bf16", group=128, k=128)


@pytest.mark.parametrize("k", [32, 64, 128, 256])
@pytest.mark.parametrize("group", [None, 0, 32, 64, 128, 256, 96])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_transforms(env, k, group, dtype):
    d = {32: 1056, 64: 960, 128: 1152, 256: 1280}[k]
    if group == 96:
        d = 768 if k == 256 else 1152
    elif group and d % group:
        d = 1280
    for n in (1, 37):
        _check(env, n, d, dtype, k=k, group=group, values="f32" if dtype == "f32" else "bf16")


@pytest.mark.parametrize("k", [0, 64])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("gain", [False, True])
@pytest.mark.parametrize("norm", [False, True])
def test_parts_left_out(env, k, residual, gain, norm):
    _check(env, 5, 320, "f32", residual=residual, gain=gain, norm=norm, k=k, group=64, values=None, offset=0.0)
    _check(env, 5, 320, "bf16", residual=residual, gain=gain, norm=norm, k=k, group=None, values="f32")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strides_and_alignments(env, dtype):
    _check(env, 6, 256, dtype, group=64, pad=16)
    _check(env, 6, 256, dtype, group=64, pad=1)          # rows at odd addresses
    _check(env, 6, 256, dtype, group=64, pad=16, k=64)
    torch, cafeq = env
    x = torch.randn((4, 257), device="cuda:0").to(torch.float32 if dtype == "f32" else torch.bfloat16)
    a = cafeq.norm_quantize(x[:, 1:], group=32)           # the first row misaligned
    b = cafeq.norm_quantize(x[:, 1:].contiguous(), group=32)
    assert torch.equal(a.codes, b.codes) and torch.equal(a.scales, b.scales)


@pytest.mark.parametrize("d", [96, 2304, 40000])
def test_the_sum_in_place(env, d):
    torch, cafeq = env
    x, r = torch.randn((3, d), device="cuda:0"), torch.randn((3, d), device="cuda:0")
    want = cafeq.norm_quantize(x, residual=r, group=32)
    for which in (0, 1):
        a, b = x.clone(), r.clone()
        got = cafeq.norm_quantize(a, residual=b, group=32, sum_out=(a, b)[which])
        assert got.sum is (a, b)[which]
        assert torch.equal(got.sum, want.sum) and torch.equal(got.codes, want.codes) and torch.equal(got.scales, want.scales)


@pytest.mark.parametrize("k", [0, 64])
def test_rows_of_zeros_tiny_and_large_numbers(env, k):
    def edit(x, r):
        x[0] = 0
        r[0] = 0
        x[1] *= 1e-30
        r[1] *= 1e-30
        x[2] *= 1e15
        r[2] *= 1e15
        x[3, :64] = 0
        r[3, :64] = 0
    o = _check(env, 5, 256, "f32", k=k, group=64, edit=edit)
    assert (o.codes[0] == 0).all() and (o.scales[0] == 0).all() and (o.values[0] == 0).all()
    assert o.scales[3, 0] == 0 and (o.scales[3, 1:] > 0).all()


def test_denormal_groups_without_a_norm(env):
    torch, cafeq = env
    x = torch.full((1, 64), 1e-41, device="cuda:0")
    x[0, 32:] = 3.0
    o = cafeq.norm_quantize(x, norm=False, group=32, values=torch.float32)
    assert torch.isfinite(o.values).all() and (o.codes[0, 32:] == 127).all()
    assert (o.values[0, :32] - 1e-41).abs().max() <= 1e-41


@pytest.mark.parametrize("k", [0, 32])
@pytest.mark.parametrize("group", [32, 0, 96])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_values_that_are_not_finite(env, bad, group, k):
    torch, cafeq = env
    x = torch.randn((4, 96), device="cuda:0")
    x[2, 40] = bad
    P = torch.eye(32, device="cuda:0").repeat(3, 1, 1) if k else None
    o = cafeq.norm_quantize(x, norm=False, Tinv=P, group=group, values=torch.float32)
    g = group or 96
    hit = torch.zeros((4, 96 // g), dtype=torch.bool, device="cuda:0")
    hit[2, 40 // g] = True
    assert torch.equal(~torch.isfinite(o.scales), hit)
    cols = hit.repeat_interleave(g, 1)
    assert (o.codes[cols] == 0).all() and torch.isfinite(o.values[~cols]).all() and not torch.isfinite(o.values[cols]).any()
    o = cafeq.norm_quantize(x, Tinv=P, group=group, values=torch.float32)   # through the norm a row takes it up as a whole or as zeros
    assert torch.isfinite(o.values[[0, 1, 3]]).all() and not torch.isfinite(o.values[2]).all()


def test_no_rows(env):
    torch, cafeq = env
    o = cafeq.norm_quantize(torch.empty((0, 64), device="cuda:0"), residual=torch.empty((0, 64), device="cuda:0"), group=32)
    assert o.codes.shape == (0, 64) and o.scales.shape == (0, 2) and o.sum.shape == (0, 64)
    P = torch.eye(32, device="cuda:0").repeat(2, 1, 1)
    assert cafeq.norm_quantize(torch.empty((0, 64), device="cuda:0"), Tinv=P, group=0).codes.shape == (0, 64)


def test_two_streams_at_once_share_nothing(env):
    torch, cafeq = env
    P = torch.linalg.qr(torch.randn((18, 128, 128)))[0].contiguous().cuda()
    xs = [torch.randn((300, 2304), device="cuda:0") for _ in range(2)]
    want = [cafeq.norm_quantize(x, Tinv=P, group=0) for x in xs]
    streams = [torch.cuda.Stream() for _ in xs]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(4):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[i].append(cafeq.norm_quantize(xs[i], Tinv=P, group=0))
    torch.cuda.synchronize()
    for i in range(2):
        for o in got[i]:
            assert torch.equal(o.codes, want[i].codes) and torch.equal(o.scales, want[i].scales)


def test_a_captured_graph_replays(env):
    torch, cafeq = env
    P = torch.linalg.qr(torch.randn((9, 128, 128)))[0].contiguous().cuda()
    codes, scales, _ = cafeq.rtn_quantize(torch.randn((300, 1152), device="cuda:0"), 4, 128)
    W = cafeq.pack_nibbles(codes, scales, 128)
    x, r, w = torch.randn((4, 1152), device="cuda:0"), torch.randn((4, 1152), device="cuda:0"), torch.randn(1152, device="cuda:0")

    def step():
        o = cafeq.norm_quantize(x, w, residual=r, Tinv=P, group=128)
        return o.sum, cafeq.infer_packed(o.codes, W, xscales=o.scales, xgroup=128)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for i in range(4):
        x.copy_(torch.randn_like(x))
        r.mul_(0.5).add_(i)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(held, step()):
            assert torch.equal(a, b)


def test_refusals(env):
    torch, cafeq = env
    dev = "cuda:0"
    x = torch.zeros((2, 64), device=dev)
    P = torch.eye(32, device=dev).repeat(2, 1, 1)
    E = cafeq.CafeqError
    for bad in (lambda: cafeq.norm_quantize(x.double()), lambda: cafeq.norm_quantize(x.cpu()), lambda: cafeq.norm_quantize(x.t()),
                lambda: cafeq.norm_quantize(x, group=48), lambda: cafeq.norm_quantize(x, group=16), lambda: cafeq.norm_quantize(x, group=-32),
                lambda: cafeq.norm_quantize(x, group=None), lambda: cafeq.norm_quantize(x, values=torch.float16),
                lambda: cafeq.norm_quantize(x, torch.zeros(63, device=dev)), lambda: cafeq.norm_quantize(x, torch.zeros(64, device=dev).double()),
                lambda: cafeq.norm_quantize(x, residual=torch.zeros((2, 63), device=dev)), lambda: cafeq.norm_quantize(x, residual=x.bfloat16()),
                lambda: cafeq.norm_quantize(x, Tinv=P[:1].contiguous()), lambda: cafeq.norm_quantize(x, Tinv=P[0]),
                lambda: cafeq.norm_quantize(x, Tinv=torch.eye(16, device=dev).repeat(4, 1, 1)), lambda: cafeq.norm_quantize(x, Tinv=P, residual=x, sum_out=x),
                lambda: cafeq.norm_quantize(torch.zeros((2, 65), device=dev)[:, 1:], Tinv=P), lambda: cafeq.norm_quantize(x, sum_out=x[:1]),
                lambda: cafeq.norm_quantize(torch.zeros((1, 65568), device=dev))):
        with pytest.raises(E):
            bad()


@pytest.mark.parametrize("k", [0, 32])
def test_rows_past_two_gigabytes(env, k):
    torch, cafeq = env
    n, d = 40000, 16384                                   # 2.6 GB of float32
    x = torch.zeros((n, d), device="cuda:0")
    at = [0, 32767, 32768, n - 1]
    x[at] = torch.randn((4, d), device="cuda:0")
    P = torch.eye(32, device="cuda:0").repeat(d // 32, 1, 1) if k else None
    o = cafeq.norm_quantize(x, Tinv=P, group=128)
    few = cafeq.norm_quantize(x[at].contiguous(), Tinv=P, group=128)
    # 1 / rms of few rows is summed in another order: scales to 64 u, and a code at a tie may move by one
    assert (o.scales[at] - few.scales).abs().max() <= 64 * U * few.scales.max()
    assert (o.codes[at].int() - few.codes.int()).abs().max() <= 1
    assert (o.codes[at] != few.codes).float().mean() <= 1e-3
    rest = torch.ones(n, dtype=torch.bool, device="cuda:0")
    rest[at] = False
    assert not o.codes[rest].any() and not o.scales[rest].any()


@pytest.mark.parametrize("k", [0, 32])
def test_operands_side_by_side_in_one_buffer(env, k):
    torch, cafeq = env
    buf = torch.randn((5, 3 * 64), device="cuda:0")
    x, r, total = buf[:, :64], buf[:, 64:128], buf[:, 128:]
    P = torch.linalg.qr(torch.randn((2, 32, 32)))[0].contiguous().cuda() if k else None
    want = cafeq.norm_quantize(x.clone(), residual=r.clone(), Tinv=P, group=32)
    got = cafeq.norm_quantize(x, residual=r, Tinv=P, group=32, sum_out=total)
    assert torch.equal(total, want.sum) and torch.equal(got.codes, want.codes) and torch.equal(got.scales, want.scales)
