"""tlc_adamw against the header's formula, bit for bit in fp32 (the CPU
reference of adamw_ref.py), and against 64 bits.

Bars of the comparison with 64 bits (U = 2^-24): m is off by 4 U (|m| + |g|)
(difference, product, sum, coefficient), v by 6 U (v + g^2); the change, a
quotient of them, by 16 U of |change| + what m's error gives it, and the new
weight by that and U |new|.
"""
import math

import numpy as np
import pytest
import torch

import adamw_ref as ref

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
RATES = dict(lr=1e-2, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.1)
U = 2.0 ** -24


def T():
    from paper_1802_07389_amd import tlc
    return tlc


@pytest.fixture(scope="module")
def ctx():
    c = T().TrainContext(max_tensors=400)
    yield c
    c.close()


def at_offset(x, offset):
    buf = torch.empty(x.numel() + offset, dtype=x.dtype, device="cuda")
    buf[offset:].copy_(x.reshape(-1))
    return buf[offset:]


def make(ctx, seed, sizes, kinds, bits, offset=0, deltas=True, sigma=1e-3):
    """A list, its gradients, and the list's states on the CPU."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    params = [at_offset((torch.randn(n, device="cuda", generator=g) * 0.02).to(
        TYPES[kinds[i % len(kinds)]]), offset) for i, n in enumerate(sizes)]
    grads = [at_offset((torch.randn(n, device="cuda", generator=g) * sigma).to(
        TYPES[kinds[(i + 1) % len(kinds)]]), offset) for i, n in enumerate(sizes)]
    states = None
    if offset:  # states at odd addresses
        nb = [-(-n // 256) for n in sizes]
        if bits == 32:
            states = [[at_offset(torch.zeros(n, device="cuda"), offset) for n in sizes]
                      for _ in range(2)]
        else:
            states = [[at_offset(torch.zeros(n, dtype=torch.uint8, device="cuda"), offset).view(t)
                       for n in sizes] for t in (torch.float8_e4m3fn, torch.float8_e5m2)]
            states.append([at_offset(torch.zeros(2 * b, device="cuda"), offset).view(b, 2)
                           for b in nb])
    out = [at_offset(torch.full((n,), 7.0, device="cuda"), offset) for n in sizes]
    return ctx.adamw_list(params, grads, bits, out if deltas else None, states)


def expected(weights, grads, t, coef=1.0, lr_scale=1.0, rates=RATES):
    """What one step has to leave: tensors on the CPU, one dict a weight."""
    f = ref.factors(t, lr_scale=lr_scale, **rates)
    done = []
    for i, p in enumerate(weights.params):
        p0, g = ref.numpy_of(p), ref.numpy_of(grads[i])
        if weights.bits == 32:
            m, v = ref.numpy_of(weights.exp_avgs[i]), ref.numpy_of(weights.exp_avg_sqs[i])
        else:
            s = weights.scales[i].cpu().numpy()
            m = ref.decode(weights.exp_avgs[i].view(torch.uint8).cpu(), torch.float8_e4m3fn, s, 0)
            v = ref.decode(weights.exp_avg_sqs[i].view(torch.uint8).cpu(), torch.float8_e5m2, s, 1)
        new, m, v = ref.fp32_step(p0, g, m, v, coef, f)
        new = ref.rounded(new, p.dtype)
        with np.errstate(all="ignore"):
            d = dict(params=new, deltas=torch.from_numpy(new.float().numpy() - p0))
        if weights.bits == 32:
            d.update(exp_avgs=torch.from_numpy(m), exp_avg_sqs=torch.from_numpy(v))
        else:
            q, w, s = ref.encode(m, v, t)
            d.update(exp_avgs=torch.from_numpy(q), exp_avg_sqs=torch.from_numpy(w),
                     scales=torch.from_numpy(s))
        done.append(d)
    return done


def same_bits(a, b):
    a = a.detach().cpu().reshape(-1)
    b = b.reshape(-1)
    if a.dtype in (torch.float8_e4m3fn, torch.float8_e5m2):
        return torch.equal(a.view(torch.uint8), b)
    both_nan = a.isnan() & b.isnan()
    word = torch.int32 if a.dtype == torch.float32 else torch.int16
    return a.dtype == b.dtype and bool(((a.view(word) == b.view(word)) | both_nan).all())


def check(weights, want):
    for i, d in enumerate(want):
        for name, x in d.items():
            if name == "deltas" and weights.deltas is None:
                continue
            assert same_bits(getattr(weights, name)[i], x), (i, name, weights.ns[i])


SIZES = {
    "one": [1], "few": [2, 3, 4, 5, 7], "blocks": [255, 256, 257, 511, 512, 513, 1023, 1025],
    "pieces": [4095, 4096, 4097, 8193], "empties": [0, 5, 0, 4096, 0], "odd": [70_001],
    "many": [(37 * i) % 3000 + 1 for i in range(150)], "none": [],
    "large": [1_500_003, 17, 900_000],
}


@pytest.mark.parametrize("sizes", SIZES)
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("kinds", [("f32",), ("bf16", "f32", "f16"), ("f16", "f16", "bf16")])
def test_steps(ctx, sizes, bits, kinds):
    for offset in (0, 1):
        w = make(ctx, 1, SIZES[sizes], kinds, bits, offset)
        for t in range(1, 5):
            want = expected(w, w.grads, t)
            ctx.adamw(w, **RATES)
            ctx.sync()
            assert int(w.step) == t
            check(w, want)
            for g in w.grads:
                g.mul_(-0.7)


@pytest.mark.parametrize("bits", [32, 8])
def test_against_64_bits(ctx, bits):
    """One step from a state in the middle of a training, in 64 bits."""
    w = make(ctx, 2, [30_001], ("f32",), bits)
    for _ in range(20):
        ctx.adamw(w, **RATES)
    t, p, g = 21, w.params[0].double(), w.grads[0].double()
    if bits == 32:
        m, v = w.exp_avgs[0].double(), w.exp_avg_sqs[0].double()
    else:
        s = w.scales[0].double().repeat_interleave(256, 0)[:30_001]
        m, v = w.exp_avgs[0].double() * s[:, 0], w.exp_avg_sqs[0].double() * s[:, 1]
    m0 = m
    m = 0.9 * m + 0.1 * g
    v = 0.99 * v + 0.01 * g * g
    hat = torch.sqrt(v / (1 - 0.99 ** t)) + 1e-8
    u = m / (1 - 0.9 ** t) / hat
    new = p - 1e-2 * (u + 0.1 * p)
    ctx.adamw(w, **RATES)
    ctx.sync()
    err_m = 4 * U * (m0.abs() + g.abs())
    bar = 1e-2 * (16 * U * (u.abs() + 0.1 * p.abs()) + err_m / (1 - 0.9 ** t) / hat) + U * new.abs()
    assert bool(((w.params[0].double() - new).abs() <= bar).all())
    assert bool(((w.deltas[0].double() - (new - p)).abs() <= bar + U * new.abs()).all())
    if bits == 32:
        assert bool(((w.exp_avgs[0].double() - m).abs() <= err_m).all())
        assert bool(((w.exp_avg_sqs[0].double() - v).abs() <= 6 * U * (v + g * g)).all())
        return
    # 8 bits: between the codes around the value, one step of the format at most
    s = w.scales[0].double().repeat_interleave(256, 0)[:30_001]
    got_m, got_v = w.exp_avgs[0].double() * s[:, 0], w.exp_avg_sqs[0].double() * s[:, 1]
    assert bool(((got_m - m).abs() <= (m.abs() / 8 + s[:, 0] * 2.0 ** -9) * (1 + 1e-5)).all())
    assert bool(((got_v - v).abs() <= (v / 4 + s[:, 1] * 2.0 ** -16) * (1 + 1e-5)).all())
    assert bool((got_v > 0).all())


def test_small_states_follow_a_slow_mean(ctx):
    """v moves by 1/1000 of its distance a step, a tenth of a percent of itself,
    where its codes are 12 % apart: the dither carries it all the same.  With a
    constant gradient v tends to its square; a state that is rounded to nearest
    would stay where it began.  Over many steps a code is off by less than one
    step of the format, 1/4 of the value, and the mean of the block by far less."""
    n = 4096
    w = make(ctx, 3, [n], ("f32",), 8)
    g = torch.linspace(0.5, 1.0, n, device="cuda")
    w.grads[0].copy_(g)
    rates = dict(RATES, beta2=0.999, lr=0.0)
    for _ in range(3000):
        ctx.adamw(w, **rates)
    w.grads[0].mul_(0.5)
    for _ in range(3000):
        ctx.adamw(w, **rates)
    ctx.sync()
    s = w.scales[0].double().repeat_interleave(256, 0)
    v = w.exp_avg_sqs[0].double() * s[:, 1]
    decay = 0.999 ** 3000
    want = (g.double() ** 2) * (1 - decay) * (decay + 0.25)
    assert bool(((v / want - 1).abs() <= 0.35).all())
    assert abs(float((v / want).mean()) - 1) <= 0.02


@pytest.mark.parametrize("bits", [32, 8])
def test_clipped_by_a_norm(ctx, bits):
    for limit in (0.0, 0.01, 1e9, math.inf):
        w = make(ctx, 4, [5000, 3, 777], ("bf16", "f32"), bits)
        r = ctx.grad_norm(w.grads)
        ctx.sync()
        norm = math.sqrt(float(r.sumsq))
        coef = np.float32(float(np.float32(limit)) / norm) if norm > limit else np.float32(1)
        want = expected(w, w.grads, 1, coef)
        ctx.adamw(w, max_norm=limit, result=r, **RATES)
        ctx.sync()
        assert np.float32(float(r.coef)) == coef and int(r.status) == 0
        assert abs(float(r.norm) - norm) <= 2 * U * norm
        check(w, want)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("count", [3, 150])
def test_step_left_out_where_the_norm_is_not_finite(ctx, bits, count):
    tlc = T()
    w = make(ctx, 5, [300 + i for i in range(count)], ("f32",), bits)
    ctx.adamw(w, **RATES)
    ctx.sync()
    names = ["params", "exp_avgs", "exp_avg_sqs"] + (["scales"] if bits == 8 else [])
    before = [[t.clone() for t in getattr(w, n)] for n in names]
    w.grads[1][7] = math.nan
    r = ctx.grad_norm(w.grads)
    ctx.adamw(w, max_norm=1.0, result=r, **RATES)
    ctx.sync()
    assert int(r.status) == tlc.TLC_E_NONFINITE and int(w.step) == 1
    for n, old in zip(names, before):
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8))
                   for a, b in zip(getattr(w, n), old))
    assert all(not bool(d.any()) for d in w.deltas)
    w.grads[1][7] = 0.5
    want = expected(w, w.grads, 2)
    ctx.adamw(w, **RATES)
    ctx.sync()
    assert int(w.step) == 2
    check(w, want)


@pytest.mark.parametrize("bits", [32, 8])
def test_extreme_gradients(ctx, bits):
    """Zeroes, subnormals, squares that overflow, NaN and infinity without a
    norm: the formula, value by value (in 8 bits their block's scale)."""
    for bad in (0.0, -0.0, 1e-38, 1e-42, 1e-20, 3e19, 1e38, math.inf, -math.inf, math.nan):
        w = make(ctx, 6, [1000], ("f32",), bits)
        w.grads[0][300] = bad
        w.grads[0][512:768] = bad
        for t in (1, 2, 3):
            want = expected(w, w.grads, t)
            ctx.adamw(w, **RATES)
            ctx.sync()
            check(w, want)


def test_rates(ctx):
    """Betas of 0, no decay, a large decay, a rate of 0, and the clock's factor."""
    for k, rates in enumerate((dict(RATES, beta1=0.0), dict(RATES, beta2=0.0),
                               dict(RATES, weight_decay=0.0), dict(RATES, lr=0.0),
                               dict(RATES, eps=1.0), dict(RATES, weight_decay=90.0))):
        for bits in (32, 8):
            w = make(ctx, 7 + k, [2000], ("f32",), bits)
            w.lr_scale.fill_(0.25)
            for t in (1, 2):
                want = expected(w, w.grads, t, lr_scale=0.25, rates=rates)
                ctx.adamw(w, **rates)
                ctx.sync()
                check(w, want)
    w = make(ctx, 9, [2000], ("f32",), 32)
    w.clock[0] = 10 ** 12  # a long training: corrections of 1
    want = expected(w, w.grads, 10 ** 12 + 1)
    ctx.adamw(w, **RATES)
    ctx.sync()
    check(w, want)
    assert int(w.step) == 10 ** 12 + 1


@pytest.mark.parametrize("bits", [32, 8])
def test_changes_in_the_gradients_place(ctx, bits):
    a, b = make(ctx, 10, [3000, 5], ("f32",), bits), make(ctx, 10, [3000, 5], ("f32",), bits)
    c = ctx.adamw_list(b.params, b.grads, bits, deltas=b.grads,
                       states=(b.exp_avgs, b.exp_avg_sqs) + ((b.scales,) if bits == 8 else ()))
    ctx.adamw(a, **RATES)
    ctx.adamw(c, **RATES)
    ctx.sync()
    assert all(torch.equal(x, y) for x, y in zip(a.deltas, b.grads))
    assert all(torch.equal(x, y) for x, y in zip(a.params, b.params))


@pytest.mark.parametrize("bits", [32, 8])
def test_many_calls_in_a_row(ctx, bits):
    """Long lists of the norm and of steps, none waited for: more of them than
    the context has places in host memory to lay a list out."""
    sizes = [(53 * i) % 900 + 1 for i in range(150)]
    w = make(ctx, 15, sizes, ("f32",), bits)
    other = make(ctx, 16, sizes[::-1], ("bf16", "f32"), bits)
    norm = math.sqrt(sum(float(g.double().square().sum()) for g in w.grads))
    state = [ref.numpy_of(p) for p in w.params]
    m = [np.zeros_like(p) for p in state]
    v = [np.zeros_like(p) for p in state]
    grads = [ref.numpy_of(g) for g in w.grads]
    results = []
    for t in range(1, 14):
        results.append(ctx.grad_norm(w.grads))
        ctx.adamw(w, **RATES)
        ctx.adamw(other, **RATES)
    ctx.sync()
    assert all(abs(float(r.norm) - norm) <= 2 * U * norm for r in results)
    for t in range(1, 14):
        f = ref.factors(t, **RATES)
        for i, g in enumerate(grads):
            state[i], m[i], v[i] = ref.fp32_step(state[i], g, m[i], v[i], 1.0, f)
            if bits == 8:
                q, c, s = ref.encode(m[i], v[i], t)
                m[i] = ref.decode(torch.from_numpy(q), torch.float8_e4m3fn, s, 0)
                v[i] = ref.decode(torch.from_numpy(c), torch.float8_e5m2, s, 1)
    assert all(same_bits(p, torch.from_numpy(x)) for p, x in zip(w.params, state))
    assert int(w.step) == int(other.step) == 13


def test_gradients_of_the_call(ctx):
    w = make(ctx, 11, [300, 40], ("f32",), 32)
    fresh = [torch.randn(300, device="cuda").bfloat16(), torch.randn(40, device="cuda")]
    want = expected(w, fresh, 1)
    ctx.adamw(w, grads=fresh, **RATES)
    ctx.sync()
    check(w, want)


@pytest.mark.parametrize("bits", [32, 8])
def test_captured_and_replayed(bits):
    """A captured step counts on and follows lr_scale; lists of more than one
    launch too; beside the program's own steps."""
    tlc = T()
    s = torch.cuda.Stream()
    with tlc.TrainContext(max_tensors=300, stream=s) as c:
        with torch.cuda.stream(s):
            w = make(c, 12, [(91 * i) % 700 + 1 for i in range(150)], ("f32", "bf16"), bits)
            r = c.norm_result()
            c.grad_norm(w.grads[:100], result=r)
            c.adamw(w, **RATES)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            c.grad_norm(w.grads[:100], result=r)
            c.adamw(w, max_norm=0.05, result=r, **RATES)
        for k in range(4):
            t = 2 + 2 * k
            with torch.cuda.stream(s):
                for x in w.grads:
                    x.mul_(-0.75)
                w.lr_scale.fill_(1.0 - 0.1 * k)
                c.grad_norm(w.grads[:100], result=r)
            torch.cuda.synchronize()
            norm = math.sqrt(float(r.sumsq))
            coef = np.float32(float(np.float32(0.05)) / norm) if norm > np.float32(0.05) else 1.0
            want = expected(w, w.grads, t, coef, lr_scale=1.0 - 0.1 * k)
            with torch.cuda.stream(s):
                g.replay()
            torch.cuda.synchronize()
            check(w, want)
            assert int(w.step) == t
            want = expected(w, w.grads, t + 1, lr_scale=1.0 - 0.1 * k)
            c.adamw(w, **RATES)
            torch.cuda.synchronize()
            check(w, want)
        c.sync()


@pytest.mark.parametrize("kinds", [("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("offset,state_offset", [(0, 0), (3, 3), (3, 1), (31, 31)])
def test_long_pieces(ctx, kinds, offset, state_offset):
    """Lists beyond the last-level cache, whose weights begin within a line, with
    their states alike or not."""
    sizes = [17_000_003, 5, 17_500_001]
    w = make(ctx, 14, sizes, kinds, 32, offset)
    if state_offset != offset:
        states = [[at_offset(torch.zeros(n, device="cuda"), state_offset) for n in sizes]
                  for _ in range(2)]
        w = ctx.adamw_list(w.params, w.grads, 32, w.deltas, states)
    want = expected(w, w.grads, 1)
    ctx.adamw(w, **RATES)
    ctx.sync()
    check(w, want)


def test_values_beyond_31_bits(ctx):
    """A tensor whose last values lie past 2^31, and their codes' dither."""
    n = (1 << 31) + 300
    zeros = dict(device="cuda")
    p = torch.zeros(n, dtype=torch.bfloat16, **zeros)
    g = torch.zeros(n, dtype=torch.bfloat16, **zeros)
    p[-300:] = 0.5
    g[-300:] = torch.randn(300, device="cuda")
    w = ctx.adamw_list([p], [g], bits=8)
    ctx.adamw(w, **RATES)
    ctx.sync()
    f = ref.factors(1, **RATES)
    p0, gr = np.full(300, 0.5, np.float32), ref.numpy_of(g[-300:])
    new, m, v = ref.fp32_step(p0, gr, np.zeros(300, np.float32), np.zeros(300, np.float32), 1.0, f)
    assert same_bits(p[-300:], ref.rounded(new, torch.bfloat16))
    first = 1 << 31  # a whole number of blocks before it
    h = [((first + k) * 0xC13FA9A9 + 0x91E10DA5) & 0xffffffff for k in range(300)]
    old = ref.dither
    try:
        ref.dither = lambda n, t: np.array(h, np.uint64)
        q, c, s = ref.encode(m, v, 1)
    finally:
        ref.dither = old
    assert same_bits(w.exp_avgs[0][-300:], torch.from_numpy(q))
    assert same_bits(w.exp_avg_sqs[0][-300:], torch.from_numpy(c))
    assert torch.equal(w.scales[0][-2:].cpu(), torch.from_numpy(s))
    assert not bool(p[:-300].view(torch.int16).any()) and not bool(w.scales[0][:-2].any())


def test_refusals(ctx):
    tlc = T()
    w = make(ctx, 13, [64], ("f32",), 32)
    e = make(ctx, 13, [64], ("f32",), 8)
    r = ctx.norm_result()
    p, g, d = w.params[0].data_ptr(), w.grads[0].data_ptr(), w.deltas[0].data_ptr()
    m, v, k = w.exp_avgs[0].data_ptr(), w.exp_avg_sqs[0].data_ptr(), w.clock.data_ptr()
    s = e.scales[0].data_ptr()
    o = dict(lr=0.1, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.0, max_norm=1.0)
    good = dict(params=[p], types=[0], ns=[64], grads=[g], grad_types=[0], state_type=0,
                exp_avgs=[m], exp_avg_sqs=[v], scales=None, deltas=[d], clock=k, result=None)
    bad = tlc.TLC_E_INVALID

    def call(options=o, **kw):
        return tlc.tlc_adamw(ctx.handle, **{**good, **kw}, options=None if options is None else
                             tlc.tlc_adamw_options(**options))

    assert call() == 0 and call(deltas=None) == 0 and call(result=r.ptr) == 0
    assert call(deltas=[g]) == 0 and call(ns=[0]) == 0
    small = dict(state_type=1, exp_avgs=[e.exp_avgs[0].data_ptr()],
                 exp_avg_sqs=[e.exp_avg_sqs[0].data_ptr()])
    assert call(**small, scales=[s]) == 0
    for kw in (dict(options=None), dict(clock=None), dict(state_type=2), dict(params=[None]),
               dict(grads=[None]), dict(exp_avgs=[None]), dict(exp_avg_sqs=[None]),
               dict(deltas=[None]), dict(types=[3]), dict(grad_types=[-1]), dict(ns=[1 << 32]),
               dict(**small, scales=[None]), dict(**small, scales=None), dict(deltas=[p]),
               dict(exp_avgs=[p]), dict(exp_avg_sqs=[m]), dict(grads=[p]), dict(clock=p),
               dict(result=m), dict(result=k), dict(deltas=[g], grad_types=[1], ns=[32]),
               dict(deltas=[g + 4])):
        assert call(**kw) == bad, kw
    many = {n: good[n] * 401 for n in ("params", "types", "ns", "grads", "grad_types", "exp_avgs",
                                       "exp_avg_sqs", "deltas")}
    assert call(**many) == bad
    assert call(**{**{n: v[:2] for n, v in many.items()}}) == bad  # the same tensor twice
    assert tlc.lib.tlc_adamw(ctx.handle, 1, None, None, None, None, None, 0, None, None, None, None,
                             tlc.ctypes.byref(tlc.tlc_adamw_options(**o)), k, None) == bad
    for name, values in (("lr", (-1.0, math.nan, math.inf)), ("beta1", (-0.1, 1.0, math.nan)),
                         ("beta2", (-0.1, 1.0, math.nan)), ("eps", (0.0, -1.0, 1e-60, math.inf)),
                         ("weight_decay", (-1.0, math.nan, math.inf))):
        for x in values:
            assert call({**o, name: x}) == bad, (name, x)
    for x in (-1.0, math.nan):
        assert call({**o, "max_norm": x}, result=r.ptr) == bad
        assert call({**o, "max_norm": x}) == 0  # not read
    ctx.sync()
    with pytest.raises(ValueError):
        ctx.adamw(w, 0.1, max_norm=1.0)
    with pytest.raises(ValueError):
        ctx.adamw(ctx.adamw_list(w.params), 0.1)
    with pytest.raises(ValueError):
        ctx.adamw(w, 0.1, grads=[w.grads[0][:5]])
    for kw in (dict(bits=16), dict(states=[w.exp_avgs]), dict(deltas=[w.params[0].bfloat16()]),
               dict(states=(w.exp_avgs, w.exp_avg_sqs), bits=8), dict(deltas=[]),
               dict(clock=torch.zeros(2, device="cuda")), dict(grads=[])):
        with pytest.raises(ValueError):
            ctx.adamw_list(w.params, **kw)
    with pytest.raises(ValueError):
        ctx.adamw_list([torch.zeros(4, 4, device="cuda").t()[:2]])
