"""tlc_embedding_grad at token counts far above a training batch's: exact sums,
and a time that grows with the tokens, not with their square.

Whole numbers whose sums stay below 2^24: every order of fp32 additions gives
them exactly.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu


def T():
    from paper_1802_07389_amd import tlc
    return tlc


def call(tokens, rows):
    """A gradient of one value a token, its ids and its table."""
    g = torch.Generator(device="cuda").manual_seed(tokens)
    ids = torch.randint(0, rows, (tokens,), device="cuda", generator=g, dtype=torch.int32)
    grad = torch.full((1, 1), 3.0, device="cuda").expand(tokens, 1)
    return grad, ids, torch.full((rows, 1), 5.0, device="cuda")


def check(ids, out, rows, start):
    want = torch.bincount(ids, minlength=rows).double() * 3.0 + start
    assert float(want.max()) < 1 << 24
    assert torch.equal(out.double().view(-1), want)


@pytest.mark.parametrize("tokens", [(1 << 18) - 1, (1 << 18) + 1, (1 << 20) + 8193, 5_000_011])
@pytest.mark.parametrize("rows", [500, 100_003, 1 << 19])
def test_sums_of_many_tokens(tokens, rows):
    with T().TrainContext(max_tokens=tokens, max_rows=rows, max_dim=1) as c:
        grad, ids, out = call(tokens, rows)
        c.embedding_grad(grad, ids, out, accumulate=True)
        c.sync()
        check(ids, out, rows, 5.0)
        c.embedding_grad(grad, ids, out)
        c.sync()
        check(ids, out, rows, 0.0)


def test_time_grows_with_the_tokens():
    """Eight times the tokens: eight times the time as the work goes, up to 2.5
    times that where caches hold less of it, and 64 times if every part of the
    tokens looked at all parts."""
    rows, times = 100_000, []
    for tokens in (1 << 24, 1 << 27):
        with T().TrainContext(max_tokens=tokens, max_rows=rows, max_dim=1) as c:
            grad, ids, out = call(tokens, rows)
            c.embedding_grad(grad, ids, out)
            c.sync()
            check(ids, out, rows, 0.0)
            best = float("inf")
            for _ in range(3):
                begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
                begin.record()
                c.embedding_grad(grad, ids, out)
                end.record()
                torch.cuda.synchronize()
                best = min(best, begin.elapsed_time(end))
            times.append(best)
            del grad, ids, out
    assert times[1] < 2.5 * 8 * times[0], times
