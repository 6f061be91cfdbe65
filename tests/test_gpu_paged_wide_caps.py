"""Caps over the paged cache that are wide against the scores: what may be off goes with the score then, not with the cap."""
import math

import numpy as np
import pytest
import torch

from oracle import scoring_ref
from paper_2411_09909_amd import binding
from tests.test_gpu_attention_masked import slopes_of
from tests.test_gpu_paged import FORMATS, allowed, bits, dev, f64, filled, host_pool

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name,H,G,D", [("amxfp4_e5m2", 8, 2, 128), ("mxfp4_e8m0", 12, 12, 64), ("amxfp4_e4m3", 16, 2, 128), ("mxfp4_round", 16, 1, 64)])
@pytest.mark.parametrize("lens,rows,max_keys", [([1, 33, 200, 64, 129], [1] * 5, 0), ([5000], [1], 5000), ([40, 7, 64, 90] * 30, [1] * 120, 90), ([300, 70], [4, 3], 0)])
@pytest.mark.parametrize("cap", [2.0 ** 20, 2.0 ** 16, 3000.0, 200.0])
def test_scores_far_below_the_cap(name, H, G, D, lens, rows, max_keys, cap):
    """As test_gpu_paged.allowed(): the size of a score alone, without the cap. The polynomial, which scores of up to a fiftieth of any cap take, is within
    2^-21.3 of a score (its constants' fit) and five roundings of 2^-24, the distance's share two more: below 2^-20 of the score, for weights and their sum."""
    rng = np.random.RandomState(int(cap) % 1000 + D)
    kind, asym = FORMATS[name]
    fmt, pool, table = filled(rng, name, G, D, 16, lens, -(-max(lens) // 16))
    starts = np.concatenate([[0], np.cumsum(rows)])
    positions = np.concatenate([np.arange(n - r, n) for n, r in zip(lens, rows)])
    q = torch.from_numpy((rng.randn(int(starts[-1]), H, D) * 0.2).astype(np.float32)).to(torch.bfloat16).cuda()
    hq, scale = f64(bits(q)).reshape(-1, H, D), 1 / math.sqrt(D)
    for slopes in (None, slopes_of(H)):
        out = binding.paged_attention(fmt, q, pool, dev(table), dev(lens), dev(starts), dev(positions), scale, max_keys=max_keys, cap=cap,
                                      slopes=None if slopes is None else torch.from_numpy(slopes).cuda())
        got = f64(bits(out)).reshape(-1, H, D)
        host = host_pool(pool)
        want, weight, _ = scoring_ref.paged_attention(hq, host, table, lens, starts, positions, scale, kind, asym, cap, slopes)
        size = scoring_ref.paged_attention(hq, host, table, lens, starts, positions, scale, kind, asym, 0.0, slopes)[2]
        bound = allowed(want, weight, size[..., None], D) + weight * 2.0 ** -19 * size[..., None]
        assert (np.abs(got - want) <= bound).all(), (np.abs(got - want) / bound).max()


def test_the_prompt_and_the_cache_agree_on_a_wide_cap():
    """The same scores either way: within the BF16 of the weights and results, whatever the cap."""
    rng = np.random.RandomState(3)
    fmt, pool, table = filled(rng, "amxfp4_e5m2", 2, 128, 16, [900, 77], 60)
    q = torch.from_numpy((rng.randn(2, 8, 128) * 0.2).astype(np.float32)).to(torch.bfloat16).cuda()
    args = (fmt, q, pool, dev(table), dev([900, 77]), dev([0, 1, 2]), dev([899, 76]), 0.1)
    plain = binding.paged_attention(*args).float()
    for cap in (2.0 ** 12, 2.0 ** 16, 2.0 ** 20):
        got = binding.paged_attention(*args, cap=cap).float()
        assert (got - plain).norm() <= 2.0 ** -8 * plain.norm(), cap
