"""tlc_embedding_grad on whole numbers, whose sums are exact.

Gradients from 1 to 7 (exact in every type), scales that are powers of two and
whole starting values: all partial sums are below 2^24, so every order of fp32
additions gives the same values, and one token that is lost, added twice or added
to another row shows, however long its run is.
"""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def T():
    from paper_1802_07389_amd import tlc
    return tlc


@pytest.fixture(scope="module")
def ctx():
    c = T().TrainContext(max_tokens=(1 << 20) + 1, max_rows=1 << 19, max_dim=1100)
    yield c
    c.close()


def make_ids(rng, kind, count, rows):
    if kind == "same":
        ids = np.full(count, rows // 2)
    elif kind == "few":
        ids = rng.integers(0, min(3, rows), count)
    elif kind == "zipf":
        ids = np.minimum(2.7 * ((rows + 2.7) / 2.7) ** rng.random(count) - 2.7, rows - 1)
    elif kind == "runs":  # runs about as long as a wave's and a block's shares of tokens
        ids = np.minimum(np.arange(count) // rng.choice([15, 16, 17, 63, 64, 65, 255, 256, 257]),
                         rows - 1)
    else:
        ids = rng.integers(0, rows, count)
    return np.ascontiguousarray(ids).astype(np.int64)


def check_exact(ctx, rng, count, rows, dim, dtype, kind, padding=None):
    ids = make_ids(rng, kind, count, rows)
    x = torch.from_numpy(rng.integers(1, 8, (count, dim)).astype(np.float32))
    keep = np.ones(count, bool) if padding is None else ids != padding
    want = torch.zeros(rows, dim, dtype=torch.float64).index_add_(
        0, torch.from_numpy(ids[keep]), x[torch.from_numpy(keep)].double())
    assert float(want.max()) < 1 << 23
    grad, at = x.to(TYPES[dtype]).cuda(), torch.from_numpy(ids).cuda()
    start = torch.from_numpy(rng.integers(-9, 10, (rows, dim)).astype(np.float32))
    for accumulate, scale in ((False, 1.0), (True, 0.5), (True, -2.0)):
        out = start.cuda()
        ctx.embedding_grad(grad, at, out, scale=scale, accumulate=accumulate,
                           padding_id=-1 if padding is None else padding)
        ctx.sync()
        exact = scale * want + (start.double() if accumulate else 0.0)
        assert torch.equal(out.cpu().double(), exact), (accumulate, scale)


@pytest.mark.parametrize("kind", ["same", "few", "zipf", "runs"])
@pytest.mark.parametrize("count", [1, 2, 65, 300, 1025, 2048, 2049, 4097, 16_385, 33_333, 65_535,
                                   65_536])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_runs_of_every_length(ctx, kind, count, dtype):
    rng = np.random.default_rng([1, count, len(kind)])
    check_exact(ctx, rng, count, 1500, 5, dtype, kind)
    check_exact(ctx, rng, count, 300, 40, dtype, kind)


@pytest.mark.parametrize("kind", ["same", "few", "zipf", "runs"])
@pytest.mark.parametrize("dim", [1, 3, 4, 255, 257, 513, 1100])
def test_rows_of_every_length(ctx, kind, dim):
    rng = np.random.default_rng([2, dim, len(kind)])
    for count in (130, 2047, 9001):
        check_exact(ctx, rng, count, 700, dim, "bf16", kind)
        check_exact(ctx, rng, count, 90, dim, "f32", kind, padding=3)


@pytest.mark.parametrize("kind", ["same", "few", "zipf", "runs"])
@pytest.mark.parametrize("count", [262_145, 300_001, (1 << 20) + 1])
def test_long_runs(ctx, kind, count):
    rng = np.random.default_rng([3, count, len(kind)])
    check_exact(ctx, rng, count, 511, 3, "f32", kind)
    check_exact(ctx, rng, count, 1 << 19, 4, "bf16", kind, padding=0)


@pytest.mark.parametrize("rows", [(1 << 27) - 1, 1 << 27, (1 << 27) + 3])
@pytest.mark.parametrize("count", [5, 700, 5000, 70_000])
@pytest.mark.parametrize("accumulate", [False, True])
def test_tables_of_2_27_rows(rows, count, accumulate):
    """Ids of 27 and 28 bits: three and four passes of the sort, in LDS and in
    memory."""
    rng = np.random.default_rng([4, count])
    ids = rng.integers(0, rows, count)
    ids[: count // 2] = rng.choice([0, 1, 511, 512, (1 << 18) - 1, 1 << 18, (1 << 26) + 5,
                                    rows - 2, rows - 1], count // 2)
    x = rng.integers(1, 8, (count, 1)).astype(np.float32)
    with T().TrainContext(max_tokens=count, max_rows=rows, max_dim=1) as c:
        out = torch.full((rows, 1), 3.0, device="cuda")
        c.embedding_grad(torch.from_numpy(x).cuda(), torch.from_numpy(ids).cuda(), out,
                         accumulate=accumulate)
        c.sync()
        at, where = np.unique(ids, return_inverse=True)
        sums = np.bincount(where, weights=x[:, 0])
        base = 3.0 if accumulate else 0.0
        at = torch.from_numpy(at).cuda()
        assert torch.equal(out[at, 0].double().cpu(), torch.from_numpy(sums) + base)
        out[at] = base
        assert bool((out == base).all())
