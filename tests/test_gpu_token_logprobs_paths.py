"""Token log probabilities on the ways that other sizes take: rows in parts in a
graph, and logits larger than the last-level cache, whole rows and parts, of every
type.  References and bars of test_gpu_token_logprobs."""
import math

import pytest
import torch

from test_gpu_token_logprobs import TYPES, T, check, rows_of, targets_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = T().TrainContext()
    yield c
    c.close()


@pytest.mark.parametrize("kind,vocab", [("f16", 140_001), ("f32", 131_072)])
def test_rows_in_parts_captured_and_replayed(kind, vocab):
    """Parts, keys and counters in the context's workspace, between eager calls
    that use them for rows of other numbers and parts."""
    s = torch.cuda.Stream()
    with T().TrainContext(stream=s) as c:
        with torch.cuda.stream(s):
            x, t = rows_of(60, 3, vocab, kind, 1), targets_of(61, 3, vocab)
            y, u = rows_of(62, 70, vocab, kind), targets_of(63, 70, vocab, ignored=0.3)
            z, w = rows_of(64, 1, 1_000_003, kind), targets_of(65, 1, 1_000_003)
            a = torch.randn(3, device="cuda")
            out, out2, d = c.token_result(3, 20), c.token_result(70, 64), torch.empty_like(x)
            c.token_logprobs(x, t, top=20, out=out)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            c.token_logprobs(x, t, top=20, out=out)
            c.token_logprobs(y, u, top=64, out=out2)
            c.token_logprobs_grad(x, t, out, a, out=d)
        last = None
        for k in range(4):
            with torch.cuda.stream(s):
                x.mul_(0.9)
                y.add_(y * 0.125)
                want = c.token_logprobs(x, t, top=20)
                other = c.token_logprobs(z, w, top=33)
                want2 = c.token_logprobs(y, u, top=64)
                grad = c.token_logprobs_grad(x, t, want, a)
                d.fill_(9.0)
                for r in (out, out2):
                    r.buffer.fill_(9.0)
                    r.top_ids.fill_(9)
                g.replay()
                again = c.token_logprobs(z, w, top=33)
            torch.cuda.synchronize()
            for got, ref in ((out, want), (out2, want2), (again, other)):
                assert torch.equal(got.buffer, ref.buffer), k
                assert torch.equal(got.top_ids, ref.top_ids)
                assert torch.equal(got.top_logprobs, ref.top_logprobs)
            assert torch.equal(d, grad)
            assert last is None or not torch.equal(out.buffer, last)
            last = out.buffer.clone()
        c.sync()


@pytest.mark.parametrize("kind,count,vocab", [
    ("f32", 200, 400_003),     # in two parts
    ("f16", 100, 1_500_001),   # in five
    ("f32", 700, 100_003), ("f16", 300, 500_009)])
def test_larger_than_the_cache(ctx, kind, count, vocab):
    """256 MiB of logits and more, at odd addresses, with masks and rows left out."""
    x = rows_of(count, count, vocab, kind, 1, 3.0, 1)
    assert count * vocab * x.element_size() >= 256 << 20
    t = targets_of(vocab, count, vocab, ignored=0.2)
    x[1::4, vocab // 2:] = -math.inf
    x[2::4, 5:vocab // 3] = torch.finfo(TYPES[kind]).min
    x[3] = -math.inf
    for top in (0, 20):
        check(ctx, x, t, 0.8, top)
