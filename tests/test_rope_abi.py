"""Argument checks of the rotary positions' entry point, which answer without touching a GPU, and the frequencies."""
import math

import pytest
import torch


@pytest.fixture(scope="module")
def luvc():
    import paper_2512_09010_b200 as luvc
    return luvc


FAKE = 4096          # an aligned address that is never dereferenced: the checks fail first


def test_the_arguments_are_checked(luvc):
    call = lambda **k: luvc.lib.luvc_rope(*[k.get(n, d) for n, d in (                                  # noqa: E731
        ("x", FAKE), ("xs", 4096), ("positions", FAKE), ("freqs", FAKE), ("tokens", 8), ("heads", 32), ("D", 128), ("rotary", 128),
        ("dtype", 0), ("out", 2 * FAKE), ("os", 4096), ("opts", None))])
    o = luvc.RopeOpts
    assert call(x=None) == 1 and call(positions=None) == 1 and call(freqs=None) == 1 and call(out=None) == 1
    assert call(dtype=2) == 7 and call(dtype=4) == 7
    assert call(tokens=-1) == 2 and call(heads=0) == 2 and call(heads=65537) == 2 and call(D=0) == 2 and call(D=1032, xs=1 << 20, os=1 << 20) == 2
    assert call(rotary=0) == 2 and call(rotary=3) == 2 and call(rotary=130) == 2
    assert call(xs=4088) == 2 and call(os=4088) == 2
    assert call(out=FAKE, os=4104) == 2                                    # in place with another stride
    assert call(opts=o(axes=65)) == 2 and call(opts=o(axes=-1)) == 2 and call(opts=o(axes=2, position_stride=-1)) == 2
    assert call(opts=o(factor=math.inf)) == 2 and call(opts=o(factor=math.nan)) == 2
    assert call(D=12, rotary=12) == 6 and call(xs=4097) == 6 and call(os=4100) == 6 and call(x=FAKE + 8) == 6 and call(out=FAKE + 2) == 6
    assert call(positions=FAKE + 2) == 6 and call(freqs=FAKE + 1) == 6 and call(opts=o(axes=2, axis=FAKE + 2)) == 6
    assert call(tokens=0, x=None, positions=None, out=None) == 0           # nothing to do


def test_the_binding_refuses_what_does_not_fit(luvc):
    with pytest.raises(ValueError):
        luvc.rope(torch.zeros(4, 2, 64, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int32), torch.ones(32))
    with pytest.raises(TypeError):
        luvc.rope(torch.zeros(4, 2, 64, dtype=torch.float16), torch.zeros(4, dtype=torch.int32), torch.ones(32))


def test_frequencies(luvc):
    f, factor = luvc.rope_frequencies(8, 10000.0)
    assert factor == 1.0 and torch.equal(f, torch.tensor([1.0, 0.1, 0.01, 0.001]))
    f, factor = luvc.rope_frequencies(8, 10000.0, stretch=4.0)
    assert factor == 1.0 and torch.equal(f, torch.tensor([0.25, 0.025, 0.0025, 0.00025]))
    f, _ = luvc.rope_frequencies(8, 10000.0, stretch=4.0, method="base")
    assert f[0] == 1.0 and float(f[-1]) == pytest.approx(0.001 / 4, rel=1e-6)
    # 4096 positions: pair i turns 4096 base^(-2 i / 64) / (2 pi) times; 32 turns at i = 10.5, one at i = 22.5
    f, factor = luvc.rope_frequencies(64, 10000.0, stretch=8.0, method="ramp", context=4096)
    plain, _ = luvc.rope_frequencies(64, 10000.0)
    assert factor == pytest.approx(0.1 * math.log(8.0) + 1.0)
    assert torch.equal(f[:11], plain[:11]) and torch.allclose(f[23:], plain[23:] / 8, rtol=1e-6, atol=0)
    middle = 10 + (23 - 10) / 2                                            # halfway: the mean of both
    want = (plain[16] + plain[17]) / 2
    assert 10 < middle < 23 and plain[17] / 8 < f[17] < want
    for bad in (dict(rotary=7), dict(rotary=0), dict(rotary=8, stretch=0.0), dict(rotary=8, method="other"), dict(rotary=8, method="ramp")):
        with pytest.raises(ValueError):
            luvc.rope_frequencies(**bad)
