"""A context that cannot be made leaves the others, and torch, working."""
import ctypes

import pytest
import torch

pytestmark = pytest.mark.gpu


def last_error():
    """What a launch made now would find, in the HIP runtime the library uses."""
    from paper_1802_07389_amd import tlc
    fn = tlc.lib.hipPeekAtLastError
    fn.restype = ctypes.c_int
    return fn()


def test_a_workspace_too_large_leaves_other_contexts_working():
    from paper_1802_07389_amd import tlc
    table = torch.arange(32.0, device="cuda").view(8, 4)
    ids = torch.tensor([3, 7, 0], device="cuda")
    out, grad = torch.empty(3, 4, device="cuda"), torch.empty(8, 4, device="cuda")
    x, residual = torch.full((1000,), 2.0, device="cuda"), torch.zeros(1000, device="cuda")
    with tlc.TrainContext(max_tokens=8, max_rows=8, max_dim=4, max_tensors=1) as ctx, \
            tlc.Context(1000) as codec:
        with pytest.raises(tlc.TLCError) as e:  # about 3 TB
            tlc.TrainContext(max_tokens=(1 << 31) - 1, max_rows=1, max_dim=10000)
        assert e.value.code == tlc.TLC_E_DEVICE and "memory" in str(e.value)
        assert last_error() == 0
        ctx.embedding(table, ids, out=out)
        ctx.embedding_grad(out, ids, grad)
        r = ctx.clip_grad_norm([x], 1.0, outs=[residual])
        ctx.sync()
        assert torch.equal(out, table[ids]) and torch.equal(grad[ids], out)
        assert float(r.coef) < 1.0
        residual.zero_()
        codec.compress(x, residual, 1.0)
        codec.sync()
