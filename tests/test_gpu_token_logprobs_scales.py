"""Token log probabilities and their gradient at scales from tiny to the largest
that the calls take, with masked entries, against the 64-bit references and bars
of test_gpu_token_logprobs.  What lies beyond fp32 is infinite there too."""
import math

import pytest
import torch

from test_gpu_token_logprobs import (IGNORE, T, TYPES, U, grad_reference, near, reference, rows_of,
                                     targets_of)

pytestmark = pytest.mark.gpu

SHAPES = [(40, 3000), (300, 40), (3, 140_001)]  # a block, a wave and several blocks a row


@pytest.fixture(scope="module")
def ctx():
    c = T().TrainContext()
    yield c
    c.close()


def close(got, want, bar):
    """near(), with what rounds to infinity in got's type infinite."""
    rounded = want.to(got.dtype).double()
    near(got, torch.where(rounded.isinf(), rounded, want), bar)


def spread(x, scale, sigma):
    """Rows of x, whose values are N(0, 1), with exponents of about N(0, sigma)."""
    x.copy_((x.double() * (sigma / scale)).to(x.dtype))


def mask(x):
    """Masked entries of either kind, a row of one entry and a row of none."""
    vocab = x.shape[1]
    x[:, vocab // 2::7] = -math.inf
    x[1::2, vocab // 3::5] = torch.finfo(x.dtype).min
    x[0] = -math.inf
    x[2] = -math.inf
    x[2, vocab // 4] = x[1, 0]


def check(ctx, x, targets, scale, top=20):
    r = ctx.token_logprobs(x, targets, scale=scale, top=top)
    ctx.sync()
    s = float(torch.tensor(scale, dtype=torch.float32))
    skip = targets == IGNORE
    ref = reference(x, targets, s)
    for name, (want, bar) in ref.items():
        bar = torch.where(skip, 0.0, bar.nan_to_num(posinf=0.0))
        close(getattr(r, name), torch.where(skip, 0.0, want), bar)
    order = torch.sort(x.float() + 0.0, dim=1, descending=True, stable=True)
    assert torch.equal(r.top_ids.long(), torch.where(skip[:, None], -1, order.indices[:, :top]))
    m, ls = ref["max"][0][:, None], ref["log_sum"][0][:, None]
    z = (order.values[:, :top].double() - m) * s
    lp = torch.where(m == -math.inf, -math.inf, z - ls)
    bar = ref["log_sum"][1][:, None].nan_to_num() + (
        (4 * z.abs() + lp.abs()) * U).nan_to_num(nan=0.0, posinf=0.0)
    close(r.top_logprobs, torch.where(skip[:, None], 0.0, lp), bar)
    return r


def check_grad(ctx, x, targets, r, a, b, scale, kind):
    s = float(torch.tensor(scale, dtype=torch.float32))
    want, bar = grad_reference(x, targets, r.buffer, a, torch.zeros_like(a) if b is None else b, s)
    got = ctx.token_logprobs_grad(x, targets, r, a, b, scale=scale, dtype=TYPES[kind])
    ctx.sync()
    info = torch.finfo(got.dtype)
    last = want.abs() * info.eps / 2 + info.smallest_normal * info.eps / 2
    # (what lies between the type's largest number and the bar around it may be either)
    most = info.max * (1 + info.eps / 4)
    either = (want.abs() + bar + last > most) & (want.abs() - bar - last < most)
    either &= (got.abs() >= info.max * (1 - info.eps)) & (got.sign() == want.sign())
    close(torch.where(either, 0.0, got), torch.where(either, 0.0, want),
          bar * (1 + info.eps) + last)
    return got


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("scale", [1e-6, 1e4, 1e10, 1e18])
@pytest.mark.parametrize("count,vocab", SHAPES)
def test_scales_and_masked_entries(ctx, kind, scale, count, vocab):
    g = torch.Generator(device="cuda").manual_seed(count)
    a, b = (torch.randn(count, device="cuda", generator=g) for _ in range(2))
    t = targets_of(vocab, count, vocab, ignored=0.2)
    for sigma in (3.0, 3.0 * scale):  # exponents, logits of that size
        x = rows_of(7, count, vocab, kind, 3, 1.0, 1)
        spread(x, scale, sigma)
        if not bool(x.isfinite().all()):
            continue  # beyond fp16
        mask(x)
        r = check(ctx, x, t, scale)
        for bonus in (None, b):
            for out in ("f32", "bf16"):
                got = check_grad(ctx, x, t, r, a, bonus, scale, out)
                assert bool(got.isfinite().all()) and bool((got[0] == 0).all())


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("scale,size", [(1e18, 1e21), (1e18, 1e25), (1e10, 1e30), (1.0, 1e37)])
@pytest.mark.parametrize("count,vocab", [(40, 3000), (300, 40)])
def test_factors_whose_product_with_the_scale_is_beyond_fp32(ctx, kind, scale, size, count, vocab):
    """scale a and scale b may be: what they are multiplied by may be small, or 0."""
    g = torch.Generator(device="cuda").manual_seed(count)
    a, b = (torch.randn(count, device="cuda", generator=g) * size for _ in range(2))
    t = targets_of(vocab, count, vocab, ignored=0.2)
    x = rows_of(8, count, vocab, kind, 0, 1.0)
    spread(x, scale, 6.0)
    mask(x)
    r = check(ctx, x, t, scale)
    for one, bonus in ((a, None), (torch.zeros_like(a), b), (a, b), (a / size, b), (a, b / size)):
        for out in ("f32", "bf16"):
            got = check_grad(ctx, x, t, r, one, bonus, scale, out)
            assert not bool(got.isnan().any())


@pytest.mark.parametrize("scale", [1e-30, 1.0, 1e18])
def test_infinite_factors(ctx, scale):
    """An infinite gradient is one at every p > 0, however small the scale."""
    x = torch.zeros(4, 100, device="cuda")
    t = torch.tensor([3, 50, 99, 0], device="cuda")
    a = torch.tensor([math.inf, -math.inf, 2.0, math.inf], device="cuda")
    r = ctx.token_logprobs(x, t, scale=scale)
    got = ctx.token_logprobs_grad(x, t, r, a, None, scale=scale)
    with_bonus = ctx.token_logprobs_grad(x, t, r, a, torch.ones_like(a), scale=scale)
    ctx.sync()
    want = torch.full_like(x, -math.inf)
    want[1] = math.inf
    want[torch.arange(4), t] = a
    for d in (got, with_bonus):
        assert torch.equal(d[[0, 1, 3]], want[[0, 1, 3]]) and bool(d[2].isfinite().all())


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("scale,factor", [(0.5, 1.0), (3e-38, 1e20)])
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("count,vocab", SHAPES)
def test_logits_further_apart_than_fp32_reaches(ctx, kind, scale, factor, masked, count, vocab):
    """Differences of logits may be beyond fp32 where their products with the scale
    are not."""
    x = rows_of(9, count, vocab, kind, 0, 1.0)
    x.copy_((x.double() * 1e38).clamp(-3e38, 3e38).to(x.dtype))
    x[:, :2] = torch.tensor([3e38, -3e38], device="cuda")
    if masked:
        x[:, vocab // 2::3] = -math.inf
    t = targets_of(vocab, count, vocab)
    t[::3] = 1
    r = check(ctx, x, t, scale)
    assert bool(r.logprob[::3].isfinite().all())
    g = torch.Generator(device="cuda").manual_seed(count)
    a, b = (torch.randn(count, device="cuda", generator=g) * factor for _ in range(2))
    for bonus in (None, b):
        check_grad(ctx, x, t, r, a, bonus, scale, "f32")
