"""A context that a program still holds when the interpreter ends."""
import pytest


@pytest.mark.parametrize("kind,destroy", [("Context", "tlc_ctx_destroy"),
                                          ("TrainContext", "tlc_train_destroy")])
def test_close_after_the_module_is_cleared(monkeypatch, kind, destroy):
    from paper_1802_07389_amd import tlc
    ctx = object.__new__(getattr(tlc, kind))
    ctx.handle = 1
    closed = []
    with monkeypatch.context() as m:
        m.setattr(tlc, destroy, None)
        ctx.close()
        m.setattr(tlc, destroy, closed.append)
        ctx.close()
        ctx.close()
    assert closed == [1] and ctx.handle is None
