"""Scores of the attention over the paged cache where the two scales of a group lie far apart: one element of one sign, large, the others
of the other sign and small, and queries that are zero or tiny on the large one's dimension. What the small ones give must not be lost
against the large scale."""
import math

import numpy as np
import pytest
import torch

from oracle import paged_ref
from paper_2411_09909_amd import binding
from tests.test_gpu_paged import FORMATS, THETA, activations, allowed, bits, dev, f64, host_pool, make_pool

pytestmark = pytest.mark.gpu

# format, exponent of the small elements' size, exponents by which the large ones exceed it (E4M3 scales: 2^-9 to 448; E5M2: 2^-16 to 57344)
CASES = [("amxfp4_e5m2", -13, 12), ("amxfp4_e5m2", -13, 20), ("amxfp4_e5m2", -13, 28), ("amxfp4_e4m3", -6, 12), ("amxfp4_e4m3", -6, 14),
         ("amxfp4_e8m0", -13, 12), ("amxfp4_e8m0", -13, 24), ("amxfp4_e8m0", -13, 40), ("amxfp4_round", -13, 24), ("mxfp4_e5m2", -3, 2)]


def lopsided(rng, shape, base, ratio, at):
    """Keys [tokens, kv_heads, D]: in each group of 32 the elements have a sign, drawn for each token and group, and a size of about
    2^base; the one of place at[group] has the other sign and is 2^ratio times as large."""
    n, G, D = shape
    sign = rng.choice([-1.0, 1.0], (n, G, D // 32, 1))
    x = np.abs(rng.randn(n, G, D // 32, 32)) * 2.0 ** base * sign
    large = -sign[..., 0] * rng.uniform(2, 4, (n, G, D // 32)) * 2.0 ** (base + ratio)
    for g, i in enumerate(at):
        x[:, :, g, i] = large[:, :, g]
    return x.reshape(shape).astype(np.float32)


def check(rng, name, base, ratio, H, G, D, lens, rows, max_keys=0, page=32):
    kind, asym = FORMATS[name]
    fmt = binding.make_format(kind, asym)
    count = [-(-n // page) for n in lens]
    ids = rng.permutation(sum(count) + 2)
    table, used = np.full((len(lens), max(count)), -1), 0
    for b, c in enumerate(count):
        table[b, :c], used = ids[used:used + c], used + c
    slots = np.concatenate([table[b, np.arange(n) // page] * page + np.arange(n) % page for b, n in enumerate(lens)])
    at = rng.randint(0, 32, D // 32)
    x = activations(rng, len(slots), (1 + 2 * G) * D)
    x[:, D:(1 + G) * D] = lopsided(rng, (len(slots), G, D), base, ratio, at).reshape(len(slots), -1)
    pool = make_pool(fmt, len(ids), G, D, page, seed=int(rng.randint(1000)))
    binding.paged_write(fmt, torch.from_numpy(x).cuda(), pool, dev(slots), dev(np.zeros(len(slots))), 1, THETA)  # (position 0: as they are)
    starts = np.concatenate([[0], np.cumsum(rows)])
    positions = np.concatenate([np.arange(n - r, n) for n, r in zip(lens, rows)])
    # scores of some 8 out of the small elements; the large one's dimension adds nothing for half of the heads, as much for the others
    q = rng.randn(len(positions), H, D // 32, 32) * 8 * 2.0 ** -base
    for g, i in enumerate(at):
        q[:, :, g, i] *= np.where(rng.rand(len(positions), H) < 0.5, 0, 2.0 ** -ratio)
    q = torch.from_numpy(q.reshape(len(positions), H, D).astype(np.float32)).to(torch.bfloat16).cuda()
    out = binding.paged_attention(fmt, q, pool, dev(table), dev(lens), dev(starts), dev(positions), 1 / math.sqrt(D), max_keys=max_keys)
    want, weight, size = paged_ref.attention(f64(bits(q)), host_pool(pool), table, lens, starts, positions, 1 / math.sqrt(D), kind, asym)
    assert size.max() > 8  # (scores that tell keys apart)
    over = np.abs(f64(bits(out)).reshape(want.shape) - want) / allowed(want, weight, size[..., None], D)
    print("%.3f of what is allowed" % over.max())
    assert over.max() <= 1, np.unravel_index(over.argmax(), over.shape)


@pytest.mark.parametrize("name,base,ratio", CASES)
@pytest.mark.parametrize("H,G,D", [(4, 1, 128), (8, 1, 128), (16, 1, 128), (4, 4, 64), (16, 1, 64)])  # four, two and one column
def test_scales_far_apart(name, base, ratio, H, G, D):
    check(np.random.RandomState(ratio + D + H), name, base, ratio, H, G, D, [1, 40, 130, 257], [1, 1, 1, 1])


@pytest.mark.parametrize("name,base,ratio", CASES)
@pytest.mark.parametrize("H,G,D,lens,rows", [(4, 1, 128, [3000], [1]), (6, 2, 64, [2100, 7], [3, 1]), (8, 8, 128, [30] * 40, [1] * 40)])
def test_scales_far_apart_split_and_by_the_wave(name, base, ratio, H, G, D, lens, rows):
    check(np.random.RandomState(ratio + D), name, base, ratio, H, G, D, lens, rows, max_keys=max(lens))
