"""Attention to an encoder's states against the formula in 64 bits.

The bound of an output element, worked out from the inputs before anything is run: scores are fp32 sums of D products (each
product and each of the at most D additions may lose 2^-23 of the largest partial sum), a factor and a bias (2^-22 of the score, 2^-23
of the bias); a weight is off by that times its own size and by 2^-21 (a power of two in fp32), in the numerator and in the denominator;
bf16: it enters its product with the values off by 2^-8; sums over t states lose 2^-23 for each at most; the result is rounded once to its type."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def luvc():
    import paper_2512_09010_b200 as luvc
    assert torch.cuda.is_available()
    luvc.check_status()
    return luvc


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def starts_of(counts, first=0):
    return ints([first + sum(counts[:i]) for i in range(len(counts) + 1)])


def inputs(dtype, hq, heads, D, queries, keys, seed=0, q_more=0, k_before=0, k_more=0):
    """Parts of wider tensors; tokens and states of no sequence are NaN."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = TYPES[dtype]
    qt, kt = sum(queries) + q_more, k_before + sum(keys) + k_more
    q = torch.randn((qt, hq + 1, D), generator=g, device="cuda").to(t)[:, :hq]
    kv = torch.randn((kt, 2 * heads, D), generator=g, device="cuda") + 1.5 * torch.randn((1, 2 * heads, D), generator=g, device="cuda")
    kv[:k_before], kv[k_before + sum(keys):] = math.nan, math.nan
    kv = kv.to(t)
    return q, kv[:, :heads], kv[:, heads:], starts_of(queries), starts_of(keys, k_before)


def check(q, k, v, qs, ks, got, lse, scale=None, bias=None):
    hq, D = q.shape[1:]
    group = hq // k.shape[1]
    scale = D ** -0.5 if scale is None else scale
    f32 = q.dtype == torch.float32
    u = 2.0 ** -24 if f32 else 2.0 ** -8
    qs, ks = qs.tolist(), ks.tolist()
    for i in range(len(ks) - 1):
        a, b, t = slice(qs[i], qs[i + 1]), slice(ks[i], ks[i + 1]), ks[i + 1] - ks[i]
        if t == 0:
            assert not got[a].any() and (lse is None or bool((lse[a] == -math.inf).all()))
            continue
        for h in range(hq):
            x, y, z = q[a, h].double(), k[b, h // group].double(), v[b, h // group].double()
            s, size = x @ y.t() * scale, x.abs() @ y.abs().t() * abs(scale)
            off = size * (D + 2) * 2.0 ** -23 + s.abs() * 2.0 ** -22
            if bias is not None:
                w = bias[b].double()
                s = s + w
                off = off + torch.where(w.isfinite(), w.abs(), 0.0) * 2.0 ** -23
                z = torch.where((w == -math.inf)[:, None], 0.0, z)
                s = torch.where(w == -math.inf, -math.inf, s)
            keep = s > -math.inf
            if not keep.any():
                assert not got[a, h].any() and (lse is None or bool((lse[a, h] == -math.inf).all()))
                continue
            top = s.amax(1, keepdim=True)
            p = torch.exp(s - top)
            total = p.sum(1, keepdim=True)
            p = p / total
            want, spread = p @ z, p @ z.abs()
            wrong = torch.where(keep, off, 0.0).amax(1, keepdim=True)
            bound = spread * (2 * wrong * 1.01 + 2.0 ** -20 + (0 if f32 else 2.0 ** -8) + (t + 64) * 2.0 ** -23)
            bound = bound * (1 + u) + u * want.abs()
            diff = (got[a, h].double() - want).abs()
            assert bool((diff <= bound).all()), (i, h, t, float((diff / bound).max()))
            if lse is not None:
                ref = (top + total.log())[:, 0]
                assert bool(((lse[a, h].double() - ref).abs() <= wrong[:, 0] + (t + 64) * 2.0 ** -23 + 2.0 ** -20 + ref.abs() * 2.0 ** -22).all())


SHAPES = [(28, 4, 128), (8, 8, 64), (12, 1, 256), (6, 3, 80), (20, 1, 48), (3, 3, 8), (4, 2, 136), (16, 2, 100), (5, 1, 16), (2, 2, 200)]
LENGTHS = [([1], [1]), ([1, 3, 0, 2], [64, 0, 17, 200]), ([9, 40, 19], [63, 128, 129]), ([200], [700]), ([1, 1, 1], [1300, 5, 400]), ([130, 1], [1, 2000])]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s)))
@pytest.mark.parametrize("lengths", LENGTHS, ids=lambda x: "x".join(map(str, x[0] + x[1]))[:24])
def test_ragged_sequences(luvc, dtype, shape, lengths):
    hq, heads, D = shape
    if dtype == "bf16" and D % 8:
        D += 4
    q, k, v, qs, ks = inputs(dtype, hq, heads, D, *lengths, seed=D, q_more=3, k_before=2, k_more=5)
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    out, lse = luvc.attn_cross(q, k, v, q_starts=qs, k_starts=ks, want_lse=True, out=out)
    assert luvc.check_status() == 0
    check(q, k, v, qs, ks, out, lse)
    assert bool((out[-3:] == 7.0).all())                        # behind the last sequence
    assert torch.equal(luvc.attn_cross(q, k, v, q_starts=qs, k_starts=ks)[:-3], out[:-3])       # the same bits


@pytest.mark.parametrize("dtype,hq,heads,D,queries,keys", [
    ("f32", 8, 2, 64, [300, 7], [5000, 3000]), ("f32", 2, 2, 128, [1], [30000]), ("bf16", 16, 4, 128, [700, 129], [5000, 16385]),
    ("bf16", 7, 1, 128, [1], [40000]), ("bf16", 4, 4, 64, [513], [3001]), ("bf16", 8, 1, 256, [100, 90], [4000, 4001]),
    ("bf16", 28, 4, 128, [1] * 60, [300] * 60), ("bf16", 2, 1, 96, [70] * 33, [130] * 33), ("f32", 2, 1, 96, [70] * 33, [130] * 33)])
def test_long_and_many(luvc, dtype, hq, heads, D, queries, keys):
    q, k, v, qs, ks = inputs(dtype, hq, heads, D, queries, keys, seed=1)
    one = all(x == 1 for x in queries)
    out, lse = luvc.attn_cross(q, k, v, q_starts=None if one else qs, k_starts=ks, want_lse=True)
    assert luvc.check_status() == 0
    check(q, k, v, qs, ks, out, lse)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_thousands_of_sequences(luvc, dtype):
    rng = torch.Generator().manual_seed(0)
    queries, keys = (torch.randint(0, n, (4096,), generator=rng).tolist() for n in (4, 9))
    q, k, v, qs, ks = inputs(dtype, 2, 1, 16, queries, keys)
    out, lse = luvc.attn_cross(q, k, v, q_starts=qs, k_starts=ks, want_lse=True)
    assert luvc.check_status() == 0
    some = list(range(0, 4096, 41)) + [4095]
    for i in some:
        check(q, k, v, qs[i:i + 2], ks[i:i + 2], out, lse)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hq,heads,D,queries", [(8, 2, 64, [40, 3]), (28, 4, 128, [1, 1]), (4, 2, 128, [200, 90]), (6, 1, 256, [10, 50])])
def test_biases_and_masks(luvc, dtype, hq, heads, D, queries):
    keys = [333, 140]
    q, k, v, qs, ks = inputs(dtype, hq, heads, D, queries, keys, seed=5)
    g = torch.Generator(device="cuda").manual_seed(1)
    sizes = torch.randint(1, 50, (473,), generator=g, device="cuda").float().log()
    low = torch.finfo(torch.float32).min
    for case in range(6):
        bias = sizes.clone()
        if case == 1:
            bias[torch.rand(473, generator=g, device="cuda") < 0.5] = -math.inf
        if case == 2:
            bias[:200], bias[333:] = -math.inf, -math.inf       # whole tiles, and a whole sequence
        if case == 3:
            bias[100:333], bias[333:] = low, low                # masks of the lowest value, and nothing else
        if case == 4:
            bias[:] = -math.inf
        if case == 5:
            bias[::2], bias[5] = -1e30, 60.0
        out, lse = luvc.attn_cross(q, k, v, q_starts=qs, k_starts=ks, key_bias=bias, want_lse=True, scale=0.2)
        assert luvc.check_status() == 0
        check(q, k, v, qs, ks, out, lse, scale=0.2, bias=bias)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hq,queries", [(4, 300), (4, 20), (2, 1)])
def test_masked_states_may_hold_anything(luvc, dtype, hq, queries):
    q, k, v, qs, ks = inputs(dtype, hq, 2, 64, [queries], [300], seed=3)
    bias = torch.zeros(300, device="cuda")
    bias[10:200], bias[290:] = -math.inf, -math.inf
    want = luvc.attn_cross(q, k, v, q_starts=qs, k_starts=ks, key_bias=bias)
    for bad in (math.nan, math.inf, -3e38):
        k[10:200], v[290:], v[12:40], k[299] = bad, bad, bad, -bad
        assert torch.equal(luvc.attn_cross(q, k, v, q_starts=qs, k_starts=ks, key_bias=bias), want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("queries,keys", [(300, 500), (3, 500), (1, 40)])
def test_infinities_and_nan_give_what_the_formula_gives(luvc, dtype, queries, keys):
    def formula(q, k, v):
        s = torch.einsum("ahd,bhd->hab", q.double(), k.double().repeat_interleave(2, 1)) / 8
        p = torch.softmax(s, dim=2)
        return (p[..., None] * v.double().repeat_interleave(2, 1).transpose(0, 1)[:, None]).sum(2).transpose(0, 1)

    for case in range(5):
        q, k, v, qs, ks = inputs(dtype, 4, 2, 64, [queries], [keys], seed=case)
        k.mul_(0.25)                                            # no weight is far below the others
        if case == 0:
            v[7, 0, 3], v[20, 1, 5], v[21, 1, 5] = math.inf, math.inf, -math.inf
        if case == 1:
            v[keys - 1, 1, 9] = math.nan
        if case == 2:
            k[3, 0, 0] = math.nan
        if case == 3:
            q[0, 1, 2] = math.nan
        if case == 4:
            v[:, 0] = 3e38                                      # sums beyond the range, results inside
        got, want = luvc.attn_cross(q, k, v, q_starts=qs, k_starts=ks).double(), formula(q, k, v)
        if case == 4:
            assert bool((got[:, :2].isfinite()).all() and ((got[:, :2] / want[:, :2]) - 1).abs().amax() < 2.0 ** -7) if dtype == "bf16" else True
            continue
        assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.isinf(), want.isinf())
        assert torch.equal(got.sign()[got.isinf()], want.sign()[got.isinf()])
        ok = want.isfinite()
        assert float((got - want)[ok].abs().max()) <= 2.0 ** -5 * float(want[ok].abs().max())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_scales(luvc, dtype):
    q, k, v, qs, ks = inputs(dtype, 4, 2, 64, [150, 4], [200, 70], seed=6)
    for scale in (-0.1, 1.0, 1e-4):
        out, lse = luvc.attn_cross(q, k, v, q_starts=qs, k_starts=ks, scale=scale, want_lse=True)
        check(q, k, v, qs, ks, out, lse, scale=scale)
    big = luvc.attn_cross(q, k, v, q_starts=qs, k_starts=ks, scale=1e4)           # one state takes it all
    s = torch.einsum("ahd,bhd->hab", q[:150].double(), k[:200].double().repeat_interleave(2, 1))
    near = s.topk(2, dim=2).values
    best = v[:200].repeat_interleave(2, 1).transpose(0, 1).gather(1, s.argmax(2)[..., None].expand(-1, -1, 64))
    clear = (near[..., 0] - near[..., 1]) > 1e-2
    # bf16 (half a step is 2^-8 of the value): the weight that is left is not quite 1, its score times 10^4 being rounded, and off by 2^-8 of
    # itself in the product but not in the sum; then the result is rounded by 2^-8 of itself: together 2^-7 (1 + 2^-9) of the value
    off = (big[:150].transpose(0, 1)[clear].double() - best[clear].double()).abs()
    assert bool((off <= best[clear].double().abs() * (0.0 if dtype == "f32" else 2.0 ** -7 * (1 + 2.0 ** -9))).all())


def test_growing_scores_bring_new_references(luvc):
    """States in the order of their scores: the maximum grows in every tile."""
    q, k, v, qs, ks = inputs("bf16", 4, 2, 128, [260], [1500], seed=7)
    k.copy_(torch.randn_like(k) * 0.02 + (torch.arange(1500, device="cuda") / 100.0)[:, None, None].to(k.dtype))
    q.copy_((q.float() * 0.05 + 0.3).to(q.dtype))
    out, lse = luvc.attn_cross(q, k, v, q_starts=qs, k_starts=ks, scale=0.5, want_lse=True)
    check(q, k, v, qs, ks, out, lse, scale=0.5)
    k.copy_(k.flip(0).clone())
    out, lse = luvc.attn_cross(q, k, v, q_starts=qs, k_starts=ks, scale=0.5, want_lse=True)
    check(q, k, v, qs, ks, out, lse, scale=0.5)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_streams_workspaces_and_graphs(luvc, dtype):
    q, k, v, qs, ks = inputs(dtype, 8, 2, 64, [100, 3], [900, 1500], seed=8)
    want = luvc.attn_cross(q, k, v, q_starts=qs, k_starts=ks)
    ws = torch.zeros(luvc.attn_cross_workspace_bytes(), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        got = luvc.attn_cross(q, k, v, q_starts=qs, k_starts=ks, workspace=ws)
    stream.synchronize()
    assert torch.equal(got, want)
    assert not ws[:1024].any()                                  # counters are zero again
    out = torch.zeros_like(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        luvc.attn_cross(q, k, v, q_starts=qs, k_starts=ks, workspace=ws, out=out)
        luvc.attn_cross(q, k, v, q_starts=qs, k_starts=ks, workspace=ws, out=out)
    q.neg_()
    k.neg_()
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_refusals_of_the_binding(luvc):
    q, k, v, qs, ks = inputs("bf16", 4, 2, 64, [3, 4], [5, 6])
    good = dict(q=q, k=k, v=v, q_starts=qs, k_starts=ks)
    assert luvc.attn_cross(**good).shape == q.shape
    bias = torch.zeros(11, device="cuda")
    for error, bad in (
        (ValueError, dict(k=k[:5])), (ValueError, dict(k_starts=ks[:2])), (ValueError, dict(q_starts=qs.long())), (ValueError, dict(k_starts=ks.cpu())),
        (ValueError, dict(key_bias=bias[:5])), (ValueError, dict(key_bias=bias.double())), (ValueError, dict(key_bias=bias.expand(2, 11))),
        (TypeError, dict(q=q.float())), (TypeError, dict(q=q.half())), (ValueError, dict(q=q.transpose(0, 1))), (ValueError, dict(q=q[..., :32])),
        (ValueError, dict(out=torch.empty_like(q, dtype=torch.float32))), (ValueError, dict(k=k.cpu(), v=v.cpu())),
        (ValueError, dict(workspace=torch.zeros(10, device="cuda")[::2])), (ValueError, dict(device_status=torch.zeros(3, dtype=torch.int32, device="cuda"))),
        (luvc.LuvcError, dict(workspace=torch.zeros(1024, dtype=torch.uint8, device="cuda"))), (luvc.LuvcError, dict(scale=math.inf)),
        (luvc.LuvcError, dict(q=torch.zeros((7, 3, 64), dtype=torch.bfloat16, device="cuda")))):
        with pytest.raises(error):
            luvc.attn_cross(**{**good, **bad})
    assert luvc.attn_cross(q[:0], k, v, q_starts=ints([0, 0, 0]), k_starts=ks).shape == (0, 4, 64)
    assert not luvc.attn_cross(q, k[:0], v[:0], q_starts=qs, k_starts=ints([0, 0, 0])).any()
    assert luvc.check_status() == 0


@pytest.mark.parametrize("hq,heads,D,queries,keys", [(8, 2, 64, [300, 20], [900, 1500]), (4, 1, 128, [1], [5000]), (4, 4, 256, [70], [300])])
def test_a_wait_that_gives_up(luvc, hq, heads, D, queries, keys):
    """A copy that is waited for in vain ends the call with a status, in milliseconds; the workspace is as it must be, the next call right."""
    q, k, v, qs, ks = inputs("bf16", hq, heads, D, queries, keys, seed=9)
    want = luvc.attn_cross(q, k, v, q_starts=qs, k_starts=ks)
    ws = torch.zeros(luvc.attn_cross_workspace_bytes(), dtype=torch.uint8, device="cuda")
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    stream = torch.cuda.current_stream().cuda_stream
    call = lambda: luvc.attn_cross(q, k, v, q_starts=qs, k_starts=ks, workspace=ws, device_status=status)       # noqa: E731
    assert torch.equal(call(), want) and luvc.read_status(status) == 0
    for _ in range(3):
        assert luvc.lib.luvc_debug_wait_probes(1, 1, status.data_ptr(), stream) == 0
        call()
        assert luvc.read_status(status) == 10
        assert luvc.lib.luvc_debug_wait_probes(0, 0, status.data_ptr(), stream) == 0
        assert not ws[:2048].any()
        assert torch.equal(call(), want) and luvc.read_status(status) == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s)))
def test_few_tokens(luvc, dtype, shape):
    """No more tokens than sequences: some have several, some none; rows of no sequence are left as they are."""
    hq, heads, D = shape
    if dtype == "bf16" and D % 8:
        D += 4
    for queries, keys, more in (([2, 0, 0, 1, 0, 0, 0, 0], [40, 0, 9, 1300, 5, 0, 64, 2], 3), ([0, 0, 5, 0, 0, 0], [1, 2, 777, 0, 3, 3], 0),
                                ([0, 1, 0, 1], [16, 0, 200, 33], 1), ([1] * 40, [37 * i % 211 for i in range(40)], 0), ([0] * 35 + [30], [3] * 35 + [500], 4)):
        q, k, v, qs, ks = inputs(dtype, hq, heads, D, queries, keys, seed=D, q_more=more, k_before=2, k_more=5)
        bias = torch.randn(k.shape[0], generator=torch.Generator().manual_seed(1)).cuda()
        bias[::5] = -math.inf
        for b in (None, bias):
            out = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
            out, lse = luvc.attn_cross(q, k, v, q_starts=qs, k_starts=ks, key_bias=b, want_lse=True, out=out)
            assert luvc.check_status() == 0
            check(q, k, v, qs, ks, out, lse, bias=b)
            assert more == 0 or bool((out[-more:] == 7.0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_thousand_single_tokens(luvc, dtype):
    keys = [(53 * i) % 300 for i in range(1024)]
    for n in (1024, 1025):                                      # in the one form and in the other
        q, k, v, qs, ks = inputs(dtype, 4, 2, 64, [1] * n, keys + [7] * (n - 1024))
        out, lse = luvc.attn_cross(q, k, v, k_starts=ks, want_lse=True)
        assert luvc.check_status() == 0
        for i in list(range(0, n, 53)) + [n - 1]:
            check(q, k, v, qs[i:i + 2], ks[i:i + 2], out, lse)
