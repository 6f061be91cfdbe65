"""Slopes so steep that one key has all the weight, in prompts and over the paged cache. Against 64 bits, as test_gpu_attention_masked."""
import math

import numpy as np
import pytest
import torch

from oracle import ref, scoring_ref
from paper_2411_09909_amd import binding
from tests.test_gpu_paged import FORMATS, bits, dev, f64, filled, host_pool

pytestmark = pytest.mark.gpu
SQ, SK = 150, 4128  # long enough for far keys to be looked for
MOST = float(np.finfo(np.float32).max)


def u16(t):
    return t.cpu().view(torch.int16).numpy().view(np.uint16)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("cap", [0.0, 20.0])
@pytest.mark.parametrize("shape", ["prompt", "far", "split", "held"])
def test_the_steepest_slopes(shape, cap, D):
    """Slopes of up to FP32's largest number, either way: the nearest key alone, or the farthest, and every number on the way is finite."""
    Sq, Sk, H = {"prompt": (70, 320, 6), "far": (SQ, SK, 184), "split": (5, 1024, 6), "held": (40, 96, 6)}[shape]
    kind, asym = ref.FP8_E5M2, 1
    gen = torch.Generator("cuda").manual_seed(D + 2)
    q, k, v = (torch.randn((n, s, D), generator=gen, device="cuda").to(torch.bfloat16) for n, s in ((H, Sq), (1, Sk), (1, Sk)))
    fmt = binding.make_format(kind, asym)
    ops = [*binding.quantize_batched(fmt, q), *binding.quantize_batched(fmt, k), *binding.quantize_batched(fmt, v, k_axis=1)]
    slopes = torch.zeros(H, device="cuda")
    slopes[:6] = torch.tensor([2.0 ** 90, -2.0 ** 90, 2.0 ** 60, MOST, -MOST, 1e30], device="cuda")
    got = binding.attention_masked(fmt, *ops, D ** -0.5, pos0=Sk - Sq, cap=cap, slopes=slopes)
    assert torch.isfinite(got).all()
    got = got.view(Sq, H, D)[:, :6].double().cpu().numpy()
    rows = [0, 3, Sq - 1]
    want, _ = scoring_ref.masked_attention(u16(q[:6]), u16(k), u16(v), D ** -0.5, True, Sk - Sq, None, None, cap, slopes[:6].cpu().numpy(), kind, asym, rows)
    # one key has all the weight, cast as 1 exactly: the result's rounding
    assert (np.abs(got - want)[rows] <= 2.0 ** -8 * np.abs(want)[rows]).all()


@pytest.mark.parametrize("name,H,G,D", [("amxfp4_e5m2", 8, 2, 128), ("mxfp4_e8m0", 6, 6, 64), ("amxfp4_e4m3", 16, 1, 64)])
@pytest.mark.parametrize("lens,rows", [([1, 33, 200, 64], [1] * 4), ([5000, 3], [1, 2])])
@pytest.mark.parametrize("cap", [0.0, 20.0])
def test_the_steepest_slopes_over_the_paged_cache(cap, lens, rows, name, H, G, D):
    kind, asym = FORMATS[name]
    rng = np.random.RandomState(D)
    fmt, pool, table = filled(rng, name, G, D, 16, lens, -(-max(lens) // 16))
    starts, positions = np.concatenate([[0], np.cumsum(rows)]), np.concatenate([np.arange(n - r, n) for n, r in zip(lens, rows)])
    q = torch.from_numpy(rng.randn(int(starts[-1]), H, D).astype(np.float32)).to(torch.bfloat16).cuda()
    slopes = np.resize([2.0 ** 90, -2.0 ** 90, 2.0 ** 60, MOST, -MOST, 1e30], H).astype(np.float32)
    got = binding.paged_attention(fmt, q, pool, dev(table), dev(lens), dev(starts), dev(positions), 1 / math.sqrt(D), cap=cap, slopes=torch.from_numpy(slopes).cuda())
    got = f64(bits(got)).reshape(-1, H, D)
    want, weight, _ = scoring_ref.paged_attention(f64(bits(q)).reshape(-1, H, D), host_pool(pool), table, lens, starts, positions, 1 / math.sqrt(D), kind, asym, cap, slopes)
    # one key has all the weight: its scale rounded to BF16 as a weight, and the result
    assert (np.abs(got - want) <= 2.0 ** -8 * weight * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(want)).all()
