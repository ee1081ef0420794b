"""Rotary positions against the formula in 64 bits.

Bound of an element, worked out before anything is run: the angle is off by 2^-23 radians and three times 2^-53 of itself (its
product with 1 / (2 pi), that product's rounding, and the 64-bit reference's own), sine and cosine by 2^-22 (two units in the last
place), the two products, their sum and the factor by 2^-24 each; the result is rounded once to its type."""
import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def luvc():
    import paper_2512_09010_b200 as luvc
    assert torch.cuda.is_available()
    return luvc


def reference(x, positions, freqs, axis=None, interleaved=False, inverse=False, factor=1.0):
    """The result and the bound of its error, without the last rounding."""
    half = freqs.numel()
    where = positions.double().view(-1, 1).expand(-1, half) if axis is None else positions.double()[axis.long()].t()
    angle = (where * freqs.double())[:, None]
    c, s = torch.cos(angle) * factor, torch.sin(angle) * (-factor if inverse else factor)
    y, x = x.double().clone(), x.double()
    bound = torch.zeros_like(y)
    a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    off = (2.0 ** -23 + 3 * 2.0 ** -53 * angle.abs() + 2.0 ** -22 + 4 * 2.0 ** -24) * abs(factor)
    bound[..., a] = bound[..., b] = (x[..., a].abs() + x[..., b].abs()) * off
    return y, bound


def check(got, want, bound):
    u = torch.finfo(got.dtype).eps / 2
    assert bool(((got.double() - want).abs() <= bound * (1 + u) + u * want.abs()).all())


def inputs(tokens, heads, D, rotary, dtype, axes=1, far=1 << 15, seed=0, wide=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((tokens, heads + wide, D), generator=g, device="cuda").to(TYPES[dtype])[:, :heads]
    shape = (axes, tokens) if axes > 1 else (tokens,)
    positions = torch.randint(-far, far, shape, generator=g, device="cuda").int()
    freqs = (10000.0 ** (-torch.arange(0, rotary, 2, device="cuda") / rotary)).float()
    axis = torch.randint(0, axes, (rotary // 2,), generator=g, device="cuda").int() if axes > 1 else None
    return x, positions, freqs, axis


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("tokens,heads,D,rotary,axes,wide", [
    (1, 1, 8, 2, 1, 0), (1, 32, 128, 128, 1, 4), (3, 5, 64, 64, 3, 1), (7, 36, 80, 40, 1, 0), (33, 12, 80, 20, 3, 2), (2, 1, 256, 256, 1, 0),
    (1000, 16, 64, 16, 1, 0), (129, 40, 128, 128, 3, 8), (5, 3, 96, 6, 2, 0), (17, 2, 1024, 1024, 1, 0), (4001, 1, 16, 12, 1, 0),
    (300, 130, 128, 96, 64, 0)])
def test_against_the_formula(luvc, dtype, interleaved, tokens, heads, D, rotary, axes, wide):
    x, positions, freqs, axis = inputs(tokens, heads, D, rotary, dtype, axes, wide=wide, seed=tokens)
    for inverse, factor in ((False, 1.0), (True, 1.25)):
        how = dict(axis=axis, interleaved=interleaved, inverse=inverse, factor=factor)
        want, bound = reference(x, positions, freqs, **how)
        check(luvc.rope(x, positions, freqs, **how), want, bound)
        work = torch.empty((tokens, heads + 3, D), dtype=x.dtype, device="cuda").fill_(7.0)       # in place, in a wider tensor
        work[:, 1:heads + 1] = x
        part = work[:, 1:heads + 1]
        assert luvc.rope(part, positions, freqs, out=part, **how) is part
        check(part, want, bound)
        assert bool((work[:, :1] == 7.0).all() and (work[:, heads + 1:] == 7.0).all())


def test_far_positions_keep_their_angles(luvc):
    x, _, freqs, _ = inputs(64, 2, 64, 64, "f32")
    positions = torch.tensor([2147483647, -2147483648, 1 << 30, 123456789, 0, 1, -1, 16777217] * 8, dtype=torch.int32, device="cuda")
    check(luvc.rope(x, positions, freqs), *reference(x, positions, freqs))


def test_the_gradient_is_the_turn_back(luvc):
    x, positions, freqs, axis = inputs(50, 3, 48, 32, "f32", axes=3, far=2000)
    for interleaved in (False, True):
        how = dict(axis=axis, interleaved=interleaved, factor=0.75)
        leaf = x.double().contiguous().requires_grad_()
        g = torch.randn(x.shape, device="cuda", dtype=torch.float64)
        half, y = freqs.numel(), leaf.clone()
        angle = (positions.double()[axis.long()].t() * freqs.double())[:, None]
        c, s = 0.75 * torch.cos(angle), 0.75 * torch.sin(angle)
        a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
        u, w = leaf[..., a], leaf[..., b]
        y = torch.zeros_like(leaf)
        y[..., a], y[..., b], y[..., 2 * half:] = u * c - w * s, u * s + w * c, leaf[..., 2 * half:]
        y.backward(g)
        got = luvc.rope(g.float(), positions, freqs, inverse=True, **how)
        _, bound = reference(g.float(), positions, freqs, inverse=True, **how)
        assert bool(((got.double() - leaf.grad).abs() <= bound + 2.0 ** -23 * (leaf.grad.abs() + g.abs())).all())
        # and against differences: <g, rope(x + h d) - rope(x - h d)> / 2 h = <grad, d>.  rope is linear, so h = 1/2 is exact but for
        # the roundings: 2^-21 of each of the sum's terms
        d = torch.randn(x.shape, device="cuda")
        difference = luvc.rope(x + d / 2, positions, freqs, **how).double() - luvc.rope(x - d / 2, positions, freqs, **how).double()
        terms = float((g.abs() * (x.double().abs() + d.double().abs()) * 2).sum())
        assert abs(float((g * difference).sum() - (got.double() * d.double()).sum())) <= 2.0 ** -21 * 2 * terms


def test_turned_and_turned_back(luvc):
    x, positions, freqs, _ = inputs(77, 4, 64, 64, "f32")
    back = luvc.rope(luvc.rope(x, positions, freqs), positions, freqs, inverse=True)
    assert float((back - x).abs().max()) <= 2.0 ** -19 * float(x.abs().max())       # two turns of 2^-21 each, of two elements


def test_axis_entries_out_of_range_and_one_row_for_all(luvc):
    x, positions, freqs, axis = inputs(9, 2, 32, 32, "f32", axes=3)
    odd = axis.clone()
    odd[0], odd[1] = -5, 99
    near = odd.clamp(0, 2)
    assert torch.equal(luvc.rope(x, positions, freqs, axis=odd), luvc.rope(x, positions, freqs, axis=near))
    same = positions[:1].expand(3, -1)
    assert torch.equal(luvc.rope(x, same, freqs, axis=axis), luvc.rope(x, positions[0], freqs))


def test_infinities_and_nan_stay_in_their_pair(luvc):
    x, positions, freqs, _ = inputs(4, 2, 32, 16, "bf16")
    clean = luvc.rope(x, positions, freqs)
    x[1, 1, 3], x[2, 0, 20] = float("nan"), float("inf")
    got = luvc.rope(x, positions, freqs)
    hit = torch.zeros_like(got, dtype=torch.bool)
    hit[1, 1, 3] = hit[1, 1, 11] = hit[2, 0, 20] = True
    assert bool(got[1, 1, 3].isnan() and got[1, 1, 11].isnan() and got[2, 0, 20].isinf())
    assert torch.equal(got[~hit], clean[~hit])


def test_nothing_to_do_and_refusals(luvc):
    x, positions, freqs, axis = inputs(6, 2, 32, 32, "bf16", axes=2)
    assert luvc.rope(x[:0], positions[0, :0], freqs).shape == (0, 2, 32)
    for bad in (dict(positions=positions[0].long()), dict(positions=positions[0, :5]), dict(positions=positions), dict(freqs=freqs.double()),
                dict(axis=axis[:3], positions=positions), dict(x=x.transpose(0, 1)), dict(out=x.float()), dict(factor=0.0),
                dict(positions=positions[0].cpu())):
        with pytest.raises(ValueError):
            luvc.rope(**{**dict(x=x, positions=positions[0], freqs=freqs), **bad})
    with pytest.raises(luvc.LuvcError):
        luvc.rope(x, positions[0], torch.ones(17, device="cuda"))                  # turns more than there is


def test_other_stream_and_captured(luvc):
    x, positions, freqs, _ = inputs(100, 8, 64, 64, "bf16")
    want = luvc.rope(x, positions, freqs)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    out = torch.zeros_like(want)
    with torch.cuda.stream(stream):
        luvc.rope(x, positions, freqs, out=out)
    stream.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        luvc.rope(x, positions, freqs, out=out)
    x.mul_(2)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want * 2)                                              # (a power of two: exact)
