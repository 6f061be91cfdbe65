"""Far keys under a slope, which the masked attention may leave out by the norms of queries and keys: keys whose squares FP32 does not hold, what
leaving keys out may cost. Against 64 bits, as test_gpu_attention_masked."""
import numpy as np
import pytest
import torch

from oracle import ref, scoring_ref
from paper_2411_09909_amd import binding

pytestmark = pytest.mark.gpu
SQ, SK = 150, 4128  # long enough for far keys to be looked for


def u16(t):
    return t.cpu().view(torch.int16).numpy().view(np.uint16)


def run(H, q, k, v, scale, slopes, kind, asym, at, rows):
    fmt = binding.make_format(kind, asym)
    ops = [*binding.quantize_batched(fmt, q), *binding.quantize_batched(fmt, k), *binding.quantize_batched(fmt, v, k_axis=1)]
    got = binding.attention_masked(fmt, *ops, scale, pos0=SK - SQ, slopes=slopes)
    assert torch.isfinite(got).all()
    one = lambda x: np.repeat(u16(x), len(at), 0)  # noqa: E731  (one key head for all)
    want, allowed = scoring_ref.masked_attention(u16(q[at]), one(k), one(v), scale, True, SK - SQ, None, None, 0.0, slopes[at].cpu().numpy(), kind, asym, rows)
    got = got.view(SQ, H, -1)[:, at].double().cpu().numpy()
    return got[rows], want[rows], allowed[rows]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kind,asym", [(ref.E8M0_FLOOR, 0), (ref.E8M0_ROUND, 1)])
@pytest.mark.parametrize("small,scale", [(-79, 85), (-76, 82), (-72, 78), (-90, 96)])
def test_keys_whose_squares_vanish(small, scale, kind, asym, D):
    """Keys of 2^-72 and less, under a scale that makes scores of thousands of them: a far key, of the first tiles, outweighs its distance."""
    H, at, rows = 184, [0, 91, 183], [0, 31, 64, SQ - 1]
    gen = torch.Generator("cuda").manual_seed(D)
    q, k = torch.ones((H, SQ, D), device="cuda").to(torch.bfloat16), torch.zeros((1, SK, D), device="cuda").to(torch.bfloat16)
    k[0, 100], k[0, 2000] = 2.0 ** small, 2.0 ** (small - 1)
    v = torch.randn((1, SK, D), generator=gen, device="cuda").to(torch.bfloat16)
    slopes = torch.full((H,), 1.5 * D / 128, device="cuda")
    got, want, allowed = run(H, q, k, v, 2.0 ** scale, slopes, kind, asym, at, rows)
    assert (np.abs(want) > 0.1).any() and (np.abs(got - want) <= allowed).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kind,asym", [(ref.E8M0_FLOOR, 0), (ref.E8M0_ROUND, 1), (ref.FP8_E5M2, 1)])
def test_large_values_of_far_keys(kind, asym, D):
    """Keys that a slope puts far below a row's sum may be left out, each by up to 2^-60 of its value: where near values are zero, or far ones larger by more
    than that, a result is so far off and no further."""
    H, at, rows = 184, [0, 1, 91, 183], [0, 31, 64, SQ - 1]
    gen = torch.Generator("cuda").manual_seed(D + 1)
    q, k, v = (torch.randn((n, s, D), generator=gen, device="cuda").to(torch.bfloat16) for n, s in ((H, SQ), (1, SK), (1, SK)))
    size = 2.0 ** 100 if kind != ref.FP8_E5M2 else 2.0 ** 14
    v[0, :1000] *= size
    v[0, 1000:, :D // 2] = 0
    slopes = torch.full((H,), 0.5, device="cuda")
    slopes[at] = torch.tensor([0.05, 0.02, 4.0, 0.0], device="cuda")
    got, want, allowed = run(H, q, k, v, D ** -0.5, slopes, kind, asym, at, rows)
    # (a weight left out is below 2^-60 of the sum, and a cast one below 2^-59: the scale of the cast is a tile's largest weight's; values are below 8 times `size`)
    assert (np.abs(got - want) <= allowed + SK * 2.0 ** -59 * 8 * size).all()
    assert (np.abs(got - want) <= allowed)[:, 3].all()  # no slope: nothing is left out
