"""Where a clipping call of the binding writes: into the outputs it is given,
also where its tensors are a list laid out before."""
import pytest
import torch


class Tensor:
    """What the binding asks of a GPU tensor."""
    is_cuda = True

    def __init__(self, n, dtype, ptr):
        self.n, self.dtype, self.ptr = n, dtype, ptr

    def numel(self):
        return self.n

    def data_ptr(self):
        return self.ptr

    def is_contiguous(self):
        return True


class Library:
    """Keeps what the last call got as outs."""

    def tlc_clip(self, *args):
        self.outs = None if args[-1] is None else list(args[-1])
        return 0

    tlc_clip_grad_norm = tlc_clip


class Result:
    ptr = 8


@pytest.fixture()
def clips(monkeypatch):
    """(the binding's list class, the two calls by outs' addresses)."""
    from paper_1802_07389_amd import tlc
    library = Library()
    monkeypatch.setattr(tlc, "lib", library)
    ctx = object.__new__(tlc.TrainContext)
    ctx.handle = None

    def clip(tensors, **outs):
        ctx.clip(tensors, 1.0, Result, **outs)
        return library.outs

    def clip_grad_norm(tensors, **outs):
        ctx.clip_grad_norm(tensors, 1.0, result=Result, **outs)
        return library.outs

    return ctx, [clip, clip_grad_norm]


def test_outs_are_used_with_and_without_a_kept_list(clips):
    ctx, calls = clips
    grads = [Tensor(5, torch.bfloat16, 64), Tensor(9, torch.float32, 128)]
    outs = [Tensor(5, torch.float32, 256), Tensor(9, torch.float32, 512)]
    own = [Tensor(5, torch.float32, 1024), Tensor(9, torch.float32, 2048)]
    for call in calls:
        assert call(grads) is None
        assert call(grads, outs=outs) == [256, 512]
        kept = ctx.tensor_list(grads)
        assert call(kept) is None
        assert call(kept, outs=outs) == [256, 512]
        assert call(kept, outs=iter(outs)) == [256, 512]
        assert call(kept) is None
        both = ctx.tensor_list(grads, own)
        assert call(both) == [1024, 2048]
        assert call(both, outs=outs) == [256, 512]
        assert call(both) == [1024, 2048]


def test_outs_of_other_sizes_or_types_are_refused(clips):
    ctx, calls = clips
    grads = [Tensor(5, torch.bfloat16, 64)]
    for tensors in (grads, ctx.tensor_list(grads)):
        for outs in ([], [Tensor(4, torch.float32, 256)], [Tensor(5, torch.bfloat16, 256)],
                     [Tensor(5, torch.float32, 256)] * 2):
            for call in calls:
                with pytest.raises(ValueError):
                    call(tensors, outs=outs)


@pytest.mark.gpu
@pytest.mark.parametrize("count", [2, 150])
def test_a_kept_list_is_clipped_into_outs(count):
    from paper_1802_07389_amd import tlc
    with tlc.TrainContext(max_tensors=count) as ctx:
        grads = [torch.full((k + 3,), 0.75, device="cuda").bfloat16() for k in range(count)]
        outs = [torch.full((k + 3,), 9.0, device="cuda") for k in range(count)]
        kept = ctx.tensor_list(grads)
        r = ctx.clip_grad_norm(kept, 1e-3, outs=outs)
        ctx.sync()
        assert float(r.coef) < 1.0
        assert all(torch.equal(o, r.coef * 0.75 * torch.ones_like(o)) for o in outs)
        for o in outs:
            o.fill_(9.0)
        ctx.clip(kept, 1e-3, ctx.grad_norm(kept), outs=outs)
        ctx.sync()
        assert all(torch.equal(o, r.coef * 0.75 * torch.ones_like(o)) for o in outs)
        assert all(bool((g == 0.75).all()) for g in grads)
