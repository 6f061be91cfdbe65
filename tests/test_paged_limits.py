"""Calls of the paged cache at the ends of what they take, refused on the host (no GPU needed)."""
import ctypes

import pytest

from paper_2411_09909_amd import binding

P = ctypes.c_void_p(0x1000)  # never dereferenced: validation fails first


@pytest.mark.parametrize("scale", [1.5 * 2.0 ** 127, 3.4e38])
def test_attention_scales_that_overflow_times_log2_e(scale):
    """They would make 0 * infinity of the largest score's exponent."""
    f = binding.make_format()
    p = binding.AmxPagedPool(16, 64, 8, 128, 0, 0x1000, 0x1000, 0x1000, 0x1000)
    assert binding.load().amxfp4_paged_attention(ctypes.byref(f), ctypes.byref(p), P, 4, 32, P, 4, 4, P, P, P, scale, 0, P, P, 1 << 40, None) == -1
    assert b"2^127" in binding.load().amxfp4_last_error()
