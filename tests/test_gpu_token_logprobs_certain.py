"""What the two calls give together for a token that is nearly certain.

The sum whose logarithm log_sum is holds the largest logit's own 1.  Each of the
additions that it goes through (three of a thread's pack and six of its wave here;
U = 2^-24) may round by U, and ln of it, near 1, and the gradient's exponent take
over that error: it is absolute, however small 1 - p is."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.mark.parametrize("above", [8.0, 14.0, 20.0, 40.0])
def test_gradient_of_a_certain_token_from_the_call_before(above):
    from paper_1802_07389_amd import tlc
    x = torch.zeros(1, 100, device="cuda")
    x[0, 3] = above
    t = torch.tensor([3], device="cuda")
    with tlc.TrainContext() as ctx:
        r = ctx.token_logprobs(x, t)
        got = ctx.token_logprobs_grad(x, t, r, torch.ones(1, device="cuda"))
        ctx.sync()
    rest = 99 * math.exp(-above)
    want = rest / (1 + rest)
    bar = 10 * U + 8 * U * want
    assert abs(float(r.log_sum) - math.log1p(rest)) <= bar
    assert abs(float(r.logprob) + math.log1p(rest)) <= bar
    assert abs(float(got[0, 3]) - want) <= bar
    others = torch.cat([got[0, :3], got[0, 4:]]).double()
    p = math.exp(-above) / (1 + rest)
    # these are relative: the exponent's error, and log_sum's
    assert bool(((others + p).abs() <= p * (5 * above + 20) * U).all())
