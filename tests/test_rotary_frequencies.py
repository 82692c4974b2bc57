"""Tables of rotary frequencies (host side, no GPU): the four ways they are scaled, from their definitions."""
import math

import pytest


@pytest.fixture(scope="module")
def cq():
    from paper_2511_19705_amd import cafeq
    return cafeq


@pytest.mark.parametrize("rot", [2, 20, 64, 128])
@pytest.mark.parametrize("scaling", ["none", "linear", "base", "parts"])
def test_definitions(cq, rot, scaling):
    freq, amplitude = cq.rotary_frequencies(rot, base=5000.0, scaling=scaling, factor=4.0, trained=1000, low=2.0, high=20.0)
    assert freq.shape == (rot // 2,)
    assert amplitude == (0.1 * math.log(4.0) + 1.0 if scaling == "parts" else 1.0)
    for i, got in enumerate(freq.tolist()):
        f = 5000.0 ** (-2 * i / rot)
        if scaling == "linear":
            f /= 4.0
        elif scaling == "base":
            f = (5000.0 * 4.0 ** (rot / max(1, rot - 2))) ** (-2 * i / rot)
        elif scaling == "parts":
            turns = 1000 * f / (2 * math.pi)
            keep = min(1.0, max(0.0, (turns - 2.0) / 18.0))
            f = keep * f + (1 - keep) * f / 4.0
        assert abs(got - f) <= 1e-14 * f


def test_ends(cq):
    plain, _ = cq.rotary_frequencies(64)
    base, _ = cq.rotary_frequencies(64, scaling="base", factor=8.0)
    assert base[0] == plain[0] and abs(base[-1] * 8.0 / plain[-1] - 1) < 1e-12
    parts, _ = cq.rotary_frequencies(64, scaling="parts", factor=8.0, trained=4096)
    assert parts[0] == plain[0] and abs(parts[-1] * 8.0 / plain[-1] - 1) < 1e-12
    for scaling in ("linear", "base", "parts"):
        same, amplitude = cq.rotary_frequencies(64, scaling=scaling, factor=1.0)
        assert amplitude == 1.0 and float((same / plain - 1).abs().max()) < 1e-14
    assert cq.rotary_frequencies(0)[0].numel() == 0


@pytest.mark.parametrize("kw", [dict(rot=3), dict(rot=-2), dict(rot=8, base=0.0), dict(rot=8, factor=0.0), dict(rot=8, scaling="other"),
                                dict(rot=8, scaling="parts", trained=0), dict(rot=8, scaling="parts", low=2.0, high=2.0)])
def test_refusals(cq, kw):
    with pytest.raises(cq.CafeqError):
        cq.rotary_frequencies(**kw)
