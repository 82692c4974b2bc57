"""The served layer of examples/serve_layer.py against the same layer in float64.

The codes' values are what the layer computes with, so the only further error is that of the activations' 8 bits and of the bfloat16
result: a group's step is its largest magnitude over 127, its rounding errors are spread evenly over a step, so with
a <= 6 standard deviations (128 Gaussian values stay below 5) the relative error is below 6 / 127 / sqrt(12) = 0.0137; bfloat16 adds 2^-9."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "serve_layer.py")


@pytest.fixture(scope="module")
def serve():
    spec = importlib.util.spec_from_file_location("serve_layer", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("tokens", [1, 7, 70])
@pytest.mark.parametrize("k,group", [(64, 64), (128, 128), (128, 32)])
def test_a_step_computes_with_the_quantized_weights(serve, tokens, k, group):
    import torch
    cafeq = serve.cafeq
    gen = torch.Generator(device="cuda:0").manual_seed(tokens + k)
    weights = [torch.randn((o, 512), generator=gen, device="cuda:0") * 0.02 for o in (96, 257)]
    T = serve.rotations(512 // k, k, gen)
    Tinv, _ = cafeq.block_inverse(T)
    packed, dense = [], []
    for w in weights:
        _, _, codes, scales = cafeq.proxy_loss_fwd_bwd(w, T, Tinv, 4, group, want_grad=False, want_codes=True)
        packed.append(cafeq.pack_nibbles(codes, scales, group))
        dense.append(codes.double() * scales.double().repeat_interleave(group, 1))
    x = torch.randn((tokens, 512), generator=gen, device="cuda:0").bfloat16()
    residual = torch.randn((tokens, 512), generator=gen, device="cuda:0").bfloat16()
    gain = torch.randn(512, generator=gen, device="cuda:0") * 0.2
    total, ys = serve.step(x, residual, gain, Tinv, packed, group)
    assert torch.equal(total, (x.float() + residual.float()).bfloat16())
    h = x.double() + residual.double()
    y = h / (h.square().mean(1, keepdim=True) + 1e-6).sqrt() * (1.0 + gain.double())
    z = torch.cat([y[:, b * k:(b + 1) * k] @ Tinv[b].double().t().contiguous() for b in range(512 // k)], 1)
    for got, w in zip(ys, dense):
        want = z @ w.t()
        assert (got.double() - want).norm() <= (0.0137 + 2.0 ** -8) * want.norm()


def test_the_example_runs_and_four_bits_are_near_the_layer(serve, capsys):
    errors = serve.main(["--d", "1024", "--outs", "512,1000", "--tokens", "3", "--steps", "3"])
    # Gaussian weights in groups of 128 on the grid of 4 bits: step = a / 7 with a < 5 deviations, 5 / 7 / sqrt(12) = 0.21
    assert len(errors) == 2 and all(e < 0.21 for e in errors)
    assert "us a step" in capsys.readouterr().out
