"""How the masked attention deals blocks of rows of unequal length out over the compute units (attention_masked.h): every block once, in turns of several
blocks that go back and forth, in a last turn that is not full, and beyond the blocks that are ranked. Sampled rows against 64 bits."""
import numpy as np
import pytest
import torch

from oracle import ref, scoring_ref
from paper_2411_09909_amd import binding

pytestmark = pytest.mark.gpu


def u16(t):
    return t.cpu().view(torch.int16).numpy().view(np.uint16)


# (32 x 2048: two turns of 8 blocks; 64 x 1504: three of 4; 40 x 1920: 6, 6 and 3; 9 x 3700: 28 and 1; 5 x 8000: 51 and 12; 2 x 17000: 133 blocks, not
# ranked; 100 x 1500: all blocks at one time, by length; 512 x 150: two blocks)
@pytest.mark.parametrize("H,S", [(32, 2048), (64, 1504), (40, 1920), (9, 3700), (5, 8000), (2, 17000), (100, 1500), (512, 150)])
@pytest.mark.parametrize("mask", ["documents", "prefixes", "causal window"])
def test_every_block_once(H, S, mask):
    D, kind, asym, Sk = 64 if H in (64, 5) else 128, ref.FP8_E5M2, 1, -(-S // 32) * 32
    rng, gen = np.random.RandomState(S), torch.Generator("cuda").manual_seed(S)
    fmt = binding.make_format(kind, asym)
    q, k, v = (torch.randn((n, s, D), generator=gen, device="cuda").to(torch.bfloat16) for n, s in ((H, S), (1, Sk), (1, Sk)))
    ops = [*binding.quantize_batched(fmt, q), *binding.quantize_batched(fmt, k), *binding.quantize_batched(fmt, v, k_axis=1)]
    first, last, causal = np.arange(S) - 199, None, mask != "prefixes"
    if mask != "causal window":
        cuts = np.unique(np.concatenate([[0], rng.randint(1, S, max(3, S // 300))]))
        lengths = np.diff(np.append(cuts, S))
        first = np.repeat(cuts, lengths)
        first = np.maximum(first, np.arange(S) - 699)  # (what the oracle walks stays short)
        if mask == "prefixes":
            last = np.maximum(np.arange(S), np.repeat(cuts + lengths * 2 // 5, lengths))
            last = np.minimum(last, np.arange(S) + 300)
            last[rng.rand(S) < 0.02] = -1
    dev = lambda a: None if a is None else torch.from_numpy(a.astype(np.int32)).cuda()  # noqa: E731
    out = torch.full((S, H * D), float("nan"), dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(binding.attention_masked_workspace_bytes(fmt, H, 1, S, Sk, D), dtype=torch.uint8, device="cuda")
    binding.attention_masked(fmt, *ops, D ** -0.5, causal=causal, first=dev(first), last=dev(last), cap=30.0, out=out, workspace=ws)
    assert torch.isfinite(out).all()
    at, rows = [0, H - 1], [min(S - 1, b + int(rng.randint(128))) for b in range(0, S, 128)]
    if len(rows) > 30:
        rows = rows[:4] + rows[4:-4:len(rows) // 12] + rows[-4:]
    want, allowed = scoring_ref.masked_attention(u16(q[at]), np.repeat(u16(k), 2, 0), np.repeat(u16(v), 2, 0), D ** -0.5, causal, 0, first, last, 30.0, None, kind, asym, rows)
    got = out.view(S, H, D)[:, at].double().cpu().numpy()
    assert (np.abs(got - want) <= allowed)[rows].all()
    # each row elsewhere as in a call of few rows (by itself, in other blocks): the same keys in the same tiles, other workgroups
    some = slice(S // 2 // 128 * 128, S // 2 // 128 * 128 + 128)
    part = binding.attention_masked(fmt, ops[0][:, some].contiguous(), ops[1][:, some].contiguous(), *ops[2:], D ** -0.5, causal=causal, pos0=some.start,
                                    first=dev(first[some]), last=None if last is None else dev(last[some]), cap=30.0)
    a, b = part.float(), out[some].float()
    assert a.shape == b.shape and (a - b).norm() <= 2.0 ** -7 * b.norm()
