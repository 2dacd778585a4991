"""tlc_adamw over lists that are laid out in other ways: more tensors
than blocks, of which a block takes several, and many tensors that are together larger
than the last-level cache.  Bit for bit against adamw_ref."""
import math

import pytest
import torch

from test_gpu_adamw import RATES, T, check, expected, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [32, 8])
def test_more_tensors_than_blocks(bits):
    tlc = T()
    count = 12_000
    sizes = [0 if i % 11 == 5 else (2500 + i % 700 if i % 97 == 3 else (i * 37) % 61 + 1)
             for i in range(count)]
    with tlc.TrainContext(max_tensors=count) as ctx:
        w = make(ctx, 21, sizes, ("f32", "bf16", "f16"), bits, 1)
        want = expected(w, w.grads, 1)
        ctx.adamw(w, **RATES)
        ctx.sync()
        assert int(w.step) == 1
        check(w, want)
        # left out: nothing changes but the deltas
        r = ctx.norm_result()
        r.sumsq.fill_(math.nan)
        names = ["params", "exp_avgs", "exp_avg_sqs"] + (["scales"] if bits == 8 else [])
        before = [torch.cat([x.reshape(-1).view(torch.uint8) for x in getattr(w, n)])
                  for n in names]
        ctx.adamw(w, max_norm=1.0, result=r, **RATES)
        ctx.sync()
        assert int(w.step) == 1 and int(r.status) == tlc.TLC_E_NONFINITE
        for n, old in zip(names, before):
            assert torch.equal(
                torch.cat([x.reshape(-1).view(torch.uint8) for x in getattr(w, n)]), old)
        assert not bool(torch.cat([d for d in w.deltas]).any())
        want = expected(w, w.grads, 2)
        ctx.adamw(w, **RATES)
        ctx.sync()
        assert int(w.step) == 2
        check(w, want)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("offset", [0, 3])
def test_many_tensors_larger_than_the_cache(bits, offset):
    """More than 64 tensors of 25 million values in all, some of a few values."""
    sizes = [5 if i % 10 == 4 else 350_000 + 1237 * i for i in range(75)]
    assert len(sizes) > 64 and sum(sizes) * 12 >= 256 << 20
    with T().TrainContext(max_tensors=len(sizes)) as ctx:
        w = make(ctx, 22, sizes, ("f32", "bf16"), bits, offset)
        for t in (1, 2):
            want = expected(w, w.grads, t)
            ctx.adamw(w, **RATES)
            ctx.sync()
            check(w, want)
