"""Capped scores of tiny scales: products of any size that FP32 holds, by far more than the cap needs. Against 64 bits, as test_gpu_attention_masked."""
import numpy as np
import pytest
import torch

from oracle import ref, scoring_ref
from paper_2411_09909_amd import binding
from tests.test_gpu_attention_fused import heads
from tests.test_gpu_attention_masked import operands, slopes_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kind,asym", [(ref.E8M0_FLOOR, 0), (ref.E8M0_ROUND, 1)])
@pytest.mark.parametrize("cap,scale,gain", [(1.0, -80, 56), (1.0, -80, 66), (1.0, -99, 75), (4.0, -76, 54), (2.0 ** -20, -110, 66), (2.0 ** 20, -62, 58), (30.0, -75, 58)])
@pytest.mark.parametrize("sloped", [False, True])
def test_large_products_and_a_tiny_scale(cap, scale, gain, sloped, kind, asym, D):
    """(The products are sums of 2^(gain + 10) at most, from below 2^-12 of what the cap takes to 2^64 and more, where their squares leave FP32's range.)"""
    Hq, Hkv, Sq, Sk = 2, 1, 40, 96
    q, k, v = heads(Hq, Sq, 1, 2.0 ** gain, D), heads(Hkv, Sk, 2, d=D), heads(Hkv, Sk, 3, d=D)
    slopes = slopes_of(Hq) if sloped else None
    want, allowed = scoring_ref.masked_attention(q, k, v, 2.0 ** scale, True, Sk - Sq, None, None, cap, slopes, kind, asym)
    fmt, ops = operands(q, k, v, kind, asym)
    got = binding.attention_masked(fmt, *ops, 2.0 ** scale, pos0=Sk - Sq, cap=cap, slopes=None if slopes is None else torch.from_numpy(slopes).cuda())
    got = got.double().cpu().numpy().reshape(Sq, Hq, D)
    assert np.isfinite(got).all() and (np.abs(got - want) <= allowed).all()
