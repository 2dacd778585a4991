"""CPU-only checks of the training-step operators' host side."""
import ctypes

import pytest


def test_calls_without_a_context_are_refused():
    from paper_1802_07389_amd import tlc
    bad = tlc.TLC_E_INVALID
    assert tlc.tlc_embedding(None, 0, 0, 1, 1, 1, 0, 0, 0, 1.0, 0, 0, 1) == bad
    assert "NULL context" in tlc.tlc_last_error_string()
    assert tlc.tlc_embedding_grad(None, 0, 0, 1, 0, 0, 0, 1, 1, 1.0, -1, 0, 1, 0) == bad
    assert tlc.tlc_grad_norm(None, [], [], [], 8) == bad
    assert tlc.tlc_clip(None, [], [], [], 1.0, 8) == bad
    assert tlc.tlc_clip_grad_norm(None, [], [], [], 1.0, 8) == bad
    assert tlc.tlc_train_sync(None) == bad
    assert tlc.tlc_train_destroy(None) == tlc.TLC_OK
    assert tlc.lib.tlc_train_create(None, 1, 1, 1, 1, None) == bad


def test_sizes_a_context_cannot_have():
    from paper_1802_07389_amd import tlc
    for args in ((1 << 31, 1, 1, 1), (1, tlc.TLC_MAX_ROWS + 1, 1, 1),
                 (1, 1, tlc.TLC_MAX_DIM + 1, 1), (1, 1, 1, tlc.TLC_MAX_TENSORS + 1)):
        with pytest.raises(tlc.TLCError) as e:
            tlc.tlc_train_create(*args, None)
        assert e.value.code == tlc.TLC_E_INVALID


def test_create_fails_cleanly_without_gpu():
    import torch
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    from paper_1802_07389_amd import tlc
    with pytest.raises(tlc.TLCError) as e:
        tlc.tlc_train_create(10, 10, 10, 10, None)
    assert e.value.code == tlc.TLC_E_DEVICE


def test_result_layout():
    from paper_1802_07389_amd import tlc
    r = tlc.tlc_norm_result
    assert ctypes.sizeof(r) == 24
    assert [r.sumsq.offset, r.norm.offset, r.coef.offset, r.status.offset] == [0, 8, 12, 16]
