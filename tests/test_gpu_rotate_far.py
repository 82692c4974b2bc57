"""GPU parity: rotary positions far from the beginning, before it, and at the ends of 32 bits, in both types and orders of pairs (tolerance as derived in
test_gpu_rotate; results of bfloat16 take the hardware's sine and cosine of the angle less its whole revolutions, good to 2^-20 of the pair, which
the 32 u = 2^-19 there hold)."""
import pytest

from tests.test_gpu_rotate import _near, _run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2511_19705_amd import cafeq
    return torch, cafeq


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("first", [0, 8192, 100_000, 8_000_000, 2 ** 31 - 50, -40, -2 ** 31])
def test_far_positions_of_both_types(env, dtype, interleaved, first):
    for d, rot in ((128, 128), (80, 20)):
        _run(env, 40, 2, 1, d, rot, dtype, interleaved=interleaved, norm=False, gain=False, first=first)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pairs_that_cancel(env, dtype):
    """x along the axis that a position turns into: one component of each pair comes out near 0, off by what sine and cosine are."""
    torch, cafeq = env
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    freq, _ = cafeq.rotary_frequencies(64, device="cuda:0")
    pos = torch.arange(1000, 1300, dtype=torch.int32, device="cuda:0")
    w = pos.double()[:, None] * freq
    x = torch.cat((torch.cos(w), -torch.sin(w)), 1)[:, None].expand(-1, 3, -1).contiguous().to(t)
    got = cafeq.rotate_heads(x, None, pos, freq)[0]
    _near(torch, got, x, pos, freq, False, False, None, 0.0, 0.0, 1.0)
