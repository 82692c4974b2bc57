"""GPU parity: norm of each head and rotary positions (cafeq_rotate_heads) against float64.

Tolerance, from the arithmetic, in units of u = 2^-24 of |y_a| + |y_b|, the normed pair: the sum of at most 512 squares is formed by eight
additions of rounded squares in a lane and six levels over lanes, 22 u at most, 11 u through the root; mean, eps, root, reciprocal and three
products add 7 u; sine and cosine of an angle good to 2^-53 of it and rounded once (pi u) are good to 2 u more; product and sum add 2 u.  All
in all below 26 u; 32 u is used.  A result of bfloat16 is off by half a step more, 2^-8 of it."""
import numpy as np
import pytest

from tests import cache_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2511_19705_amd import cafeq
    return torch, cafeq


def _near(torch, got, x, positions, freq, interleaved, norm, gain, eps, offset, amplitude):
    want, y = R.rotate(x.float().cpu().numpy(), positions.cpu().numpy(), freq.cpu().numpy(), interleaved, norm, None if gain is None else gain.cpu().numpy(),
                       eps, offset, amplitude)
    half = freq.numel()
    pair = np.abs(y)
    if half:
        a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
        s = (np.abs(y[:, :, a]) + np.abs(y[:, :, b])) * max(amplitude, 1.0)
        pair[:, :, a], pair[:, :, b] = s, s
    tol = pair * 32 * 2.0 ** -24 + 1e-37
    if x.dtype == torch.bfloat16:
        tol = tol + np.abs(want) * 2.0 ** -8
    err = np.abs(got.double().cpu().numpy() - want)
    assert (err <= tol).all(), float((err - tol).max())


def _run(env, n, hq, h, d, rot, dtype, interleaved=False, norm=True, gain=True, first=0, amplitude=1.0, fused=True, seed=0, pad=0):
    torch, cafeq = env
    gen = torch.Generator(device="cuda:0").manual_seed(seed)
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    if fused:
        x = (torch.randn((n, (hq + 2 * h) * d + pad), generator=gen, device="cuda:0") * 3).to(t)
        q, k = x[:, :hq * d].view(n, hq, d) if n < 2 or pad == 0 else x[:, :hq * d].unflatten(1, (hq, d)), x[:, hq * d:(hq + h) * d].unflatten(1, (h, d))
    else:
        q, k = (torch.randn((m, n, d), generator=gen, device="cuda:0").to(t).transpose(0, 1) for m in (hq, h))
    positions = torch.arange(first, first + n, dtype=torch.int32, device="cuda:0")
    freq, _ = cafeq.rotary_frequencies(rot, device="cuda:0")
    gq, gk = (torch.randn(d, generator=gen, device="cuda:0") for _ in range(2)) if gain else (None, None)
    keep = q.clone(), k.clone()
    oq, ok = cafeq.rotate_heads(q, k, positions, freq, interleaved=interleaved, norm=norm, gain_q=gq, gain_k=gk, gain_offset=1.0, amplitude=amplitude)
    assert torch.equal(q, keep[0]) and torch.equal(k, keep[1])
    for got, y, g in ((oq, q, gq), (ok, k, gk)):
        _near(torch, got, y, positions, freq, interleaved, norm, g, 1e-6, 1.0, amplitude)
    return q, k, positions, freq, oq, ok


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,rot", [(2, 2), (6, 4), (16, 16), (64, 64), (80, 20), (80, 32), (96, 96), (128, 128), (128, 64), (200, 56), (256, 256),
                                   (256, 0), (258, 130), (512, 512), (512, 128)])
def test_head_sizes(env, dtype, interleaved, d, rot):
    for n in (1, 5):
        _run(env, n, 6, 3, d, rot, dtype, interleaved, seed=d + rot + n)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hq,h", [(1, 1), (8, 4), (33, 11), (32, 16), (130, 1)])
def test_heads_and_many_tokens(env, dtype, hq, h):
    for n in (1, 3, 255, 300):
        _run(env, n, hq, h, 64, 64, dtype, seed=n)


@pytest.mark.parametrize("norm,gain", [(False, False), (True, False), (True, True)])
@pytest.mark.parametrize("fused,pad", [(True, 0), (True, 1), (True, 8), (False, 0)])
def test_norms_and_strides(env, norm, gain, fused, pad):
    for dtype in ("f32", "bf16"):
        _run(env, 7, 4, 2, 64, 32, dtype, norm=norm, gain=gain, fused=fused, pad=pad, amplitude=1.2)


@pytest.mark.parametrize("first", [0, 100_000, 8_000_000, 2 ** 31 - 50, -40])
def test_far_positions(env, first):
    _run(env, 40, 2, 1, 128, 128, "f32", norm=False, gain=False, first=first)


def test_one_part_and_results_in_place(env):
    torch, cafeq = env
    q, k, pos, freq, oq, ok = _run(env, 9, 4, 2, 128, 64, "bf16", norm=True, gain=False)
    assert torch.equal(cafeq.rotate_heads(q, None, pos, freq, norm=True, gain_offset=1.0)[0], oq)
    assert torch.equal(cafeq.rotate_heads(None, k, pos, freq, norm=True, gain_offset=1.0)[1], ok)
    a, b = cafeq.rotate_heads(q, k, pos, freq, norm=True, gain_offset=1.0, out_q=q, out_k=k)
    assert a is q and b is k and torch.equal(q, oq) and torch.equal(k, ok)


def test_only_the_results_are_written(env):
    torch, cafeq = env
    buf = torch.full((6, 5, 128), 7.0, device="cuda:0")
    x = torch.randn((6, 3, 64), device="cuda:0")
    freq, _ = cafeq.rotary_frequencies(64, device="cuda:0")
    pos = torch.arange(6, dtype=torch.int32, device="cuda:0")
    cafeq.rotate_heads(x, None, pos, freq, out_q=buf[:, 1:4, 32:96])
    assert torch.equal(buf[:, 1:4, 32:96], cafeq.rotate_heads(x, None, pos, freq)[0])
    buf[:, 1:4, 32:96] = 7.0
    assert (buf == 7.0).all()


def test_infinities_and_zeros_stay_in_their_head(env):
    torch, cafeq = env
    x = torch.randn((3, 4, 64), device="cuda:0")
    freq, _ = cafeq.rotary_frequencies(64, device="cuda:0")
    pos = torch.arange(3, dtype=torch.int32, device="cuda:0")
    want = cafeq.rotate_heads(x, None, pos, freq, norm=True)[0]
    y = x.clone()
    y[0, 1, 3], y[1, 2, 60], y[2, 0] = float("inf"), float("nan"), 0.0
    got = cafeq.rotate_heads(y, None, pos, freq, norm=True)[0]
    assert torch.isnan(got[0, 1]).any() and torch.isnan(got[1, 2]).all() and (got[2, 0] == 0).all()
    keep = torch.ones((3, 4), dtype=torch.bool, device="cuda:0")
    keep[0, 1] = keep[1, 2] = keep[2, 0] = False
    assert torch.equal(got[keep], want[keep])


def test_no_tokens_and_another_stream(env):
    torch, cafeq = env
    freq, _ = cafeq.rotary_frequencies(32, device="cuda:0")
    empty = torch.empty((0, 2, 32), device="cuda:0")
    assert cafeq.rotate_heads(empty, None, torch.empty(0, dtype=torch.int32, device="cuda:0"), freq)[0].shape == (0, 2, 32)
    x = torch.randn((50, 2, 32), device="cuda:0")
    pos = torch.arange(50, dtype=torch.int32, device="cuda:0")
    want = cafeq.rotate_heads(x, None, pos, freq)[0]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = cafeq.rotate_heads(x, None, pos, freq)[0]
    side.synchronize()
    assert torch.equal(got, want)
