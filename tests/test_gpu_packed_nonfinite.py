"""Products with packed 4-bit weights where an activation or a scale is not finite, however many tokens there are and whatever the groups are: an infinite
activation gives what the sum as it is written gives, an infinity of the right sign where one term is infinite and no other fails; a scale that is not finite
leaves nothing finite in its row, or its token, and touches no other."""
import pytest

pytestmark = pytest.mark.gpu
INF = float("inf")
# (tokens, rows, columns): few tokens, and as many as run in tiles; the last 128 columns are not all there
FEW, MANY = (3, 50), (700, 1147)


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2511_19705_amd import cafeq
    return torch, cafeq


def _weight(torch, rows, cols, group):
    """Codes without a zero, which times an infinity would be no number."""
    gen = torch.Generator(device="cuda:0").manual_seed(rows + cols)
    codes = torch.randint(1, 8, (rows, cols), generator=gen, device="cuda:0", dtype=torch.int8)
    codes = torch.where(torch.rand((rows, cols), generator=gen, device="cuda:0") < 0.5, -codes, codes).to(torch.int8)
    return codes, torch.rand((rows, cols // (group or cols)), generator=gen, device="cuda:0") + 0.5


@pytest.mark.parametrize("n,rows", [FEW, MANY])
@pytest.mark.parametrize("cols,group", [(1184, 32), (1248, 96), (1216, 64), (1280, 128), (1184, 0)])
@pytest.mark.parametrize("x_type", ["bf16", "f32"])
def test_an_infinite_activation(env, x_type, cols, group, n, rows):
    torch, cafeq = env
    codes, scales = _weight(torch, rows, cols, group)
    x = torch.randn((n, cols), generator=torch.Generator(device="cuda:0").manual_seed(1), device="cuda:0")
    at = [40, cols - 1, 70]                         # of tokens 0, 1 and 2: the third has no number there
    x[0, at[0]], x[1, at[1]], x[2, at[2]] = INF, -INF, float("nan")
    Y = cafeq.infer_packed(x.bfloat16() if x_type == "bf16" else x, cafeq.pack_nibbles(codes, scales, group))
    assert torch.equal(Y[0], torch.sign(codes[:, at[0]].float()) * INF)
    assert torch.equal(Y[1], torch.sign(codes[:, at[1]].float()) * -INF)
    assert bool(torch.isnan(Y[2]).all()) and bool(torch.isfinite(Y[3:]).all())


@pytest.mark.parametrize("n,rows", [FEW, MANY, (20, 300)])
@pytest.mark.parametrize("cols,group", [(1184, 32), (1248, 96), (1216, 64), (1280, 128), (1184, 0)])
@pytest.mark.parametrize("x_type", ["i8", "bf16", "f32"])
def test_scales_that_are_not_finite_stay_in_their_rows(env, x_type, cols, group, n, rows):
    torch, cafeq = env
    codes, scales = _weight(torch, rows, cols, group)
    scales[7, -1], scales[11, 0] = INF, float("nan")
    x, xs = torch.rand((n, cols), generator=torch.Generator(device="cuda:0").manual_seed(1), device="cuda:0") + 0.5, None
    if x_type == "i8":
        x, xs = (x * 40).to(torch.int8), torch.ones((n, 1), device="cuda:0")
    elif x_type == "bf16":
        x = x.bfloat16()
    bad = torch.zeros(rows, dtype=torch.bool, device="cuda:0")
    bad[[7, 11]] = True
    Y = cafeq.infer_packed(x, cafeq.pack_nibbles(codes, scales, group), xscales=xs)
    assert torch.equal(torch.isfinite(Y), ~bad.expand(n, rows))


@pytest.mark.parametrize("n,rows", [FEW, MANY, (20, 300)])
@pytest.mark.parametrize("cols,group", [(1184, 32), (1248, 96), (1216, 64), (1280, 128), (1184, 0)])
def test_scales_of_activations_that_are_not_finite_stay_with_their_tokens(env, cols, group, n, rows):
    # as a group that holds an infinity leaves them: codes 0, that scale
    torch, cafeq = env
    codes, scales = _weight(torch, rows, cols, group)
    x = torch.randint(1, 50, (n, cols), generator=torch.Generator(device="cuda:0").manual_seed(1), device="cuda:0", dtype=torch.int8)
    xs = torch.ones((n, cols // (group or cols)), device="cuda:0")
    xs[1, -1], xs[2, 0] = INF, float("nan")
    x[1, cols - (group or cols):] = 0
    x[2, :group or cols] = 0
    bad = torch.zeros((n, 1), dtype=torch.bool, device="cuda:0")
    bad[1:3] = True
    Y = cafeq.infer_packed(x, cafeq.pack_nibbles(codes, scales, group), xscales=xs, xgroup=group)
    assert torch.equal(torch.isfinite(Y), ~bad.expand(n, rows))
