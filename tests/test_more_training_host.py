"""CPU-only checks of the loss's and the optimizer's host side."""
import ctypes

import numpy as np
import pytest
import torch

import adamw_ref as ref


def test_calls_without_a_context_are_refused():
    from paper_1802_07389_amd import tlc
    bad = tlc.TLC_E_INVALID
    assert tlc.tlc_token_logprobs(None, 8, 0, 1, 4, 4, 1.0, 8, 1, -100, 8) == bad
    assert "NULL context" in tlc.tlc_last_error_string()
    assert tlc.tlc_token_logprobs_grad(None, 8, 0, 1, 4, 4, 1.0, 8, 1, -100, 8, 8, None, 8, 0,
                                       4) == bad
    options = tlc.tlc_adamw_options(0.1, 0.9, 0.99, 1e-8, 0.0, 0.0)
    assert tlc.tlc_adamw(None, [8], [0], [1], [8], [0], 0, [8], [8], None, None, options, 8) == bad


def test_struct_layouts():
    from paper_1802_07389_amd import tlc
    r, c, o = tlc.tlc_token_result, tlc.tlc_adamw_clock, tlc.tlc_adamw_options
    assert ctypes.sizeof(r) == 16 and [r.logprob.offset, r.entropy.offset, r.max.offset,
                                       r.log_sum.offset] == [0, 4, 8, 12]
    assert ctypes.sizeof(c) == 16 and [c.step.offset, c.lr_scale.offset] == [0, 8]
    assert ctypes.sizeof(o) == 48 and o.max_norm.offset == 40


@pytest.mark.parametrize("dtype,mantissa,lowest,most", [
    (torch.float8_e4m3fn, 3, -6, 126), (torch.float8_e5m2, 2, -14, 123)])
def test_reference_codes_are_the_formats_neighbours(dtype, mantissa, lowest, most):
    """The reference's codes: every code's own value gets that code whatever the
    dither, a value between two codes gets the upper one with its share of the
    dithers."""
    bits = 23 - mantissa
    codes = np.arange(most + 1, dtype=np.uint8)
    values = torch.from_numpy(codes).view(dtype).float().numpy()
    assert values[-1] == torch.finfo(dtype).max
    top = (1 << bits) - 1
    for h in (0, 1, top // 2, top):
        got = ref._codes(values, np.full(values.size, h, np.int64), bits, mantissa, lowest, most)
        assert np.array_equal(got, codes)
    for share in (0.125, 0.5, 0.75):
        mid = (values[:-1] + (values[1:] - values[:-1]) * np.float32(share)).astype(np.float32)
        h = np.linspace(0, top, 64).astype(np.int64)
        got = np.stack([ref._codes(mid, np.full(mid.size, x, np.int64), bits, mantissa, lowest,
                                   most) for x in h])
        assert np.all((got == codes[:-1]) | (got == codes[1:]))
        up = (got == codes[1:]).mean(0)
        assert np.all(np.abs(up - share) <= 1 / 32)


def test_dither_is_spread_evenly():
    """Of any 64 neighbours, and of any 64 steps of one value, every eighth of
    [0, 1) has its share: five to eleven of them."""
    for series in (ref.dither(64, 5), ref.dither(4160, 9)[4096:],
                   np.concatenate([ref.dither(8, t)[7:] for t in range(100, 164)])):
        counts = np.bincount((series >> np.uint64(29)).astype(int), minlength=8)
        assert counts.min() >= 5 and counts.max() <= 11
