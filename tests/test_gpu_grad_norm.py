"""tlc_grad_norm, tlc_clip and tlc_clip_grad_norm against 64-bit references.

Bars.  The norm and the coefficient are one rounding to fp32 (2^-24 of the
value) off what 64-bit sums give, which are off by less than 2^-40; sumsq
itself is within 2^-40.  The clipped values are bit for bit the product of the
coefficient that the call reports, rounded once.
"""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ROUND = 2.0 ** -24 * (1 + 2.0 ** -10)


def T():
    from paper_1802_07389_amd import tlc
    return tlc


@pytest.fixture(scope="module")
def ctx():
    c = T().TrainContext(max_tensors=1000)
    yield c
    c.close()


def at_offset(x, offset):
    buf = torch.empty(x.numel() + offset, dtype=x.dtype, device="cuda")
    buf[offset:].copy_(x)
    return buf[offset:]


def tensors_of(seed, sizes, kinds, sigma=1e-3, offsets=(0,)):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [at_offset((torch.randn(n, device="cuda", generator=g) * sigma).to(
        TYPES[kinds[i % len(kinds)]]), offsets[i % len(offsets)]) for i, n in enumerate(sizes)]


def sumsq_of(tensors):
    return math.fsum(float(t.double().square().sum()) for t in tensors)


def near(got, want, tol):
    return abs(float(got) - want) <= tol * abs(want)


def bits_equal(a, b):
    word = torch.int32 if a.dtype == torch.float32 else torch.int16
    return a.dtype == b.dtype and torch.equal(a.contiguous().view(word),
                                              b.contiguous().view(word))


SIZES = {
    "one": [1], "three": [3], "odd": [12345], "empties": [0, 5, 0, 0, 4096, 0],
    "edges": [4095, 4096, 4097, 8191, 8193, 1, 2, 7, 8, 9, 255, 256, 257],
    "many": [(37 * i) % 5000 + 1 for i in range(1000)], "large": [9_000_001, 17, 2_500_000],
}


@pytest.mark.parametrize("sizes", SIZES)
@pytest.mark.parametrize("kinds", [("f32",), ("bf16",), ("f16",), ("bf16", "f32", "f16")])
@pytest.mark.parametrize("offsets", [(0,), (1,), (0, 3, 2, 1, 5)])
def test_norm_and_clip(ctx, sizes, kinds, offsets):
    ts = tensors_of(1, SIZES[sizes], kinds, 0.5, offsets)
    want = sumsq_of(ts)
    r = ctx.grad_norm(ts)
    ctx.sync()
    assert near(r.sumsq, want, 2.0 ** -40) and near(r.norm, math.sqrt(want), ROUND)
    assert float(r.coef) == 1.0 and int(r.status) == 0
    first = float(r.sumsq)
    for share in (0.5, 0.999, 2.0):
        limit = float(np.float32(share * math.sqrt(want)))
        coef = min(1.0, limit / math.sqrt(want))
        outs = [at_offset(torch.full((t.numel(),), 9.0), offsets[-1]) for t in ts]
        r = ctx.clip_grad_norm(ts, limit, outs=outs)
        ctx.sync()
        assert float(r.sumsq) == first  # the same sums in the same order
        assert near(r.norm, math.sqrt(want), ROUND) and near(r.coef, coef, ROUND)
        for t, o in zip(ts, outs):
            assert bits_equal(o, r.coef * t.float())
        # in place, each in its own type
        mine = [at_offset(t, o) for t, o in zip(ts, offsets * len(ts))]
        r2 = ctx.clip_grad_norm(mine, limit)
        ctx.sync()
        assert float(r2.coef) == float(r.coef)
        for t, o in zip(ts, mine):
            assert bits_equal(o, (r.coef * t.float()).to(t.dtype))


def test_clip_in_two_calls_as_over_ranks(ctx):
    """Two shards: their sums of squares are added between the calls."""
    a, b = tensors_of(2, [5000, 70001], ("bf16",)), tensors_of(3, [123, 40000], ("f32",))
    want = sumsq_of(a + b)
    ra, rb = ctx.grad_norm(a), ctx.grad_norm(b)
    total = ra.sumsq + rb.sumsq
    ra.sumsq.copy_(total)
    rb.sumsq.copy_(total)
    outs = [torch.empty(t.numel(), device="cuda") for t in a]
    before = [t.clone() for t in b]
    limit = 0.25 * math.sqrt(want)
    ctx.clip(a, limit, ra, outs=outs)
    ctx.clip(b, limit, rb)
    ctx.sync()
    for r in (ra, rb):
        assert near(r.sumsq, want, 2.0 ** -40) and near(r.norm, math.sqrt(want), ROUND)
        assert near(r.coef, float(np.float32(limit)) / math.sqrt(want), ROUND)
    assert float(ra.coef) == float(rb.coef)
    assert all(bits_equal(o, ra.coef * t.float()) for t, o in zip(a, outs))
    assert all(bits_equal(t, rb.coef * o) for t, o in zip(b, before))


def test_extreme_values(ctx):
    """Squares that no fp32 sum holds: 1e30 and 1e-30, and fp16's ends."""
    big = torch.full((100_000,), 1e30, device="cuda")
    x = float(big[0])
    r = ctx.clip_grad_norm([big], 1.0)
    ctx.sync()
    norm = x * math.sqrt(1e5)
    assert near(r.norm, norm, ROUND) and near(r.coef, 1.0 / norm, ROUND) and int(r.status) == 0
    tiny = torch.full((100_000,), 1e-30, device="cuda")
    r = ctx.grad_norm([tiny])
    ctx.sync()
    assert near(r.norm, float(tiny[0]) * math.sqrt(1e5), ROUND)
    ends = torch.tensor([65504.0, -65504.0, 2.0 ** -24, 0.0], device="cuda").half()
    r = ctx.grad_norm([ends])
    ctx.sync()
    assert near(r.norm, 65504.0 * math.sqrt(2.0), ROUND)
    top = torch.full((3,), 3.4e38, device="cuda")  # the norm is above fp32's largest value
    out = torch.empty(3, device="cuda")
    r = ctx.clip_grad_norm([top], 3.0e38, outs=[out])
    ctx.sync()
    assert float(r.norm) == math.inf and int(r.status) == 0
    assert near(r.coef, float(np.float32(3.0e38)) / (float(top[0]) * math.sqrt(3.0)), ROUND)
    assert bits_equal(out, r.coef * top)


def test_zero_gradients_and_no_tensors(ctx):
    z = torch.zeros(7777, device="cuda")
    for limit in (0.0, 1.0):
        r = ctx.clip_grad_norm([z], limit)
        ctx.sync()
        assert float(r.norm) == 0.0 and float(r.coef) == 1.0 and not z.any()
    for ts in ([], [torch.empty(0, device="cuda")]):
        r = ctx.grad_norm(ts)
        ctx.sync()
        assert float(r.norm) == 0.0 and float(r.sumsq) == 0.0 and int(r.status) == 0
        r = ctx.clip_grad_norm(ts, 1.0)
        ctx.sync()
        assert float(r.norm) == 0.0 and float(r.coef) == 1.0
    x = torch.randn(100, device="cuda")
    r = ctx.clip_grad_norm([x], 0.0)
    ctx.sync()
    assert float(r.coef) == 0.0 and not x.any()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_nonfinite_values_write_nothing(ctx, bad, kind):
    tlc = T()
    ts = tensors_of(4, [10, 300_000, 77], (kind,))
    ts[1][250_000] = bad
    keep = [t.clone() for t in ts]
    outs = [torch.full((t.numel(),), 3.0, device="cuda") for t in ts]
    for o in (outs, None):
        r = ctx.clip_grad_norm(ts, 1e-3, outs=o)
        ctx.sync()
        assert int(r.status) == tlc.TLC_E_NONFINITE and math.isnan(float(r.coef))
        assert not math.isfinite(float(r.norm)) and not math.isfinite(float(r.sumsq))
    assert all(bits_equal(a, b) for a, b in zip(ts, keep))
    assert all(bool((o == 3.0).all()) for o in outs)
    r = ctx.grad_norm(ts)
    ctx.sync()
    assert int(r.status) == tlc.TLC_E_NONFINITE


def test_lists_kept_over_steps_and_back_to_back(ctx):
    """Calls in a row without a wait between them: each sees its own list and
    its tensors' values of the moment."""
    lists = [tensors_of(10 + k, [100 * k + 1, 5000, 60_000 + k], ("f32", "bf16")) for k in range(7)]
    kept = [ctx.tensor_list(ts) for ts in lists]
    for step in range(3):
        got = [ctx.grad_norm(ls) for ls in kept]
        ctx.sync()
        for ts, r in zip(lists, got):
            assert near(r.norm, math.sqrt(sumsq_of(ts)), ROUND)
        for ts in lists:
            ts[1].mul_(1.5)


def test_clip_into_itself_and_offsets_past_32_bits(ctx):
    """outs may be the fp32 tensors themselves; a tensor of more than 2^31
    values (in bytes beyond 2^33)."""
    ts = tensors_of(5, [1000, 33333], ("f32",))
    keep = [t.clone() for t in ts]
    r = ctx.clip_grad_norm(ts, 0.5 * math.sqrt(sumsq_of(ts)), outs=ts)
    ctx.sync()
    assert all(bits_equal(t, r.coef * k) for t, k in zip(ts, keep))
    n = (1 << 31) + 4097
    x = torch.zeros(n, device="cuda")
    x[0], x[1 << 31], x[n - 1] = 3.0, 4.0, 12.0
    r = ctx.clip_grad_norm([x], 6.5)
    ctx.sync()
    assert float(r.norm) == 13.0 and float(r.coef) == 0.5
    assert [float(x[0]), float(x[1 << 31]), float(x[n - 1])] == [1.5, 2.0, 6.0]
    assert int(x.count_nonzero()) == 3


def test_other_stream():
    s = torch.cuda.Stream()
    with T().TrainContext(max_tensors=4, stream=s) as c:
        with torch.cuda.stream(s):
            ts = tensors_of(6, [3_000_000, 10], ("bf16",))
            r = c.grad_norm(ts)
        c.sync()
        assert near(r.norm, math.sqrt(sumsq_of(ts)), ROUND)


def test_thousands_of_tensors():
    """More tensors than blocks: a block takes several pieces."""
    sizes = [(53 * i) % 700 + 1 for i in range(5000)]
    with T().TrainContext(max_tensors=5000) as c:
        flat = tensors_of(9, [sum(sizes)], ("f32",), 0.1)[0]
        ts = list(torch.split(flat, sizes))
        half = flat.bfloat16()
        mixed = [h if i % 3 else t for i, (t, h) in enumerate(zip(ts, torch.split(half, sizes)))]
        want = sumsq_of([torch.cat([m.float() for m in mixed])])
        r = c.grad_norm(mixed)
        c.sync()
        assert near(r.sumsq, want, 2.0 ** -40) and near(r.norm, math.sqrt(want), ROUND)
        out = torch.empty_like(flat)
        r = c.clip_grad_norm(mixed, 0.3 * math.sqrt(want), outs=list(torch.split(out, sizes)))
        c.sync()
        assert bits_equal(out, torch.cat([r.coef * m.float() for m in mixed]))
        before = flat.clone()
        for k in range(11):  # more calls than staging slots, without a wait
            r = c.clip_grad_norm(ts, 1e-3 * 0.5 ** k)
        c.sync()
        assert near(r.norm, 1e-3 * 0.5 ** 9, 1e-4)
        assert torch.allclose(flat, before * (1e-3 * 0.5 ** 10 / float(before.double().norm())),
                              rtol=1e-4, atol=0.0)


def test_capture():
    """A captured norm and clip follow their tensors' new values, with eager
    calls between the replays; longer lists refuse to be captured."""
    tlc = T()
    s = torch.cuda.Stream()
    with tlc.TrainContext(max_tensors=500, stream=s) as c:
        with torch.cuda.stream(s):
            ts = tensors_of(7, [50_000, 3, 70_001], ("bf16", "f32"))
            outs = [torch.empty(t.numel(), device="cuda") for t in ts]
            many = c.tensor_list(tensors_of(8, [10] * 129, ("f32",)))
            r, other = c.norm_result(), c.norm_result()
            kept = c.tensor_list(ts, outs)
            c.clip_grad_norm(kept, 0.1, result=r)
            c.grad_norm(many, result=other)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            c.clip_grad_norm(kept, 0.1, result=r)
            with pytest.raises(tlc.TLCError) as e:
                c.grad_norm(many, result=other)
        assert e.value.code == tlc.TLC_E_INVALID
        for k in range(4):
            with torch.cuda.stream(s):
                for t in ts:
                    t.mul_(1.25)
                c.grad_norm(many, result=other)
                for o in outs:
                    o.fill_(float("nan"))
                g.replay()
            torch.cuda.synchronize()
            want = math.sqrt(sumsq_of(ts))
            assert near(r.norm, want, ROUND), k
            assert near(r.coef, min(1.0, float(np.float32(0.1)) / want), ROUND)
            assert all(bits_equal(o, r.coef * t.float()) for t, o in zip(ts, outs))


def test_refusals(ctx):
    tlc = T()
    x, y = torch.randn(64, device="cuda"), torch.randn(64, device="cuda")
    res = ctx.norm_result()

    def code(fn, *args):
        return fn(ctx.handle, *args)

    p, q = x.data_ptr(), y.data_ptr()
    assert code(tlc.tlc_grad_norm, [p], [0], [64], res.ptr) == 0
    bad = tlc.TLC_E_INVALID
    assert code(tlc.tlc_grad_norm, [p], [0], [64], None) == bad
    assert code(tlc.tlc_grad_norm, [None], [0], [64], res.ptr) == bad
    assert code(tlc.tlc_grad_norm, [p], [3], [64], res.ptr) == bad
    assert code(tlc.tlc_grad_norm, [p], [0], [1 << 32], res.ptr) == bad
    assert code(tlc.tlc_grad_norm, [p], [0], [64], p + 8) == bad  # the result inside a tensor
    assert code(tlc.tlc_grad_norm, [p] * 1001, [0] * 1001, [1] * 1001, res.ptr) == bad
    assert tlc.lib.tlc_grad_norm(ctx.handle, 1, None, None, None, res.ptr) == bad
    assert tlc.tlc_grad_norm(None, [p], [0], [64], res.ptr) == bad
    assert code(tlc.tlc_grad_norm, [p, p], [0, 0], [64, 32], res.ptr) == 0  # read only
    for fn in (tlc.tlc_clip, tlc.tlc_clip_grad_norm):
        assert code(fn, [p], [0], [64], 1.0, res.ptr, [q]) == 0
        for limit in (-1.0, float("nan"), float("inf")):
            assert code(fn, [p], [0], [64], limit, res.ptr, [q]) == bad
        assert code(fn, [p], [0], [64], 1.0, None, [q]) == bad
        assert code(fn, [p], [0], [64], 1.0, res.ptr, [None]) == bad
        assert code(fn, [p, p + 64], [0, 0], [64, 8], 1.0, res.ptr) == bad  # both written
        assert code(fn, [p], [0], [32], 1.0, res.ptr, [p + 64]) == bad  # into itself, shifted
        assert code(fn, [p], [1], [64], 1.0, res.ptr, [p]) == bad  # bf16 into its own place
        assert code(fn, [p, q], [0, 0], [64, 64], 1.0, res.ptr, [q, p]) == bad
    ctx.sync()
    with pytest.raises(ValueError):
        ctx.grad_norm([x.double()])
    with pytest.raises(ValueError):
        ctx.grad_norm([x.cpu()])
    with pytest.raises(ValueError):
        ctx.grad_norm([x[::2]])
    with pytest.raises(ValueError):
        ctx.clip_grad_norm([x], 1.0, outs=[y[:5]])
    with pytest.raises(ValueError):
        ctx.clip_grad_norm([x], 1.0, outs=[y.bfloat16()])
