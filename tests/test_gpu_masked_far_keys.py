"""Far keys under a slope, which the masked attention may leave out by the norms of queries and keys: keys whose squares FP32 does not hold.
Against 64 bits, as test_gpu_attention_masked."""
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
