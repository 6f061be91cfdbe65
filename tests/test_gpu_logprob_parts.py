"""Rows of logits that are read in parts although there are a thousand of them: long ones up to 1500, and any that are too long for one part."""
import numpy as np
import pytest
import torch

from oracle import scoring_ref
from paper_2411_09909_amd import binding
from tests.test_gpu_token_logprobs import logits_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,vocab,dtype,parts", [(1100, 70000, torch.float32, True), (1500, 70000, torch.float32, True), (1501, 70000, torch.float32, False),
                                                    (1024, 600000, torch.bfloat16, True), (1600, 600000, torch.bfloat16, True), (1100, 30000, torch.bfloat16, False)])
@pytest.mark.parametrize("top,cap", [(20, 0.0), (1, 30.0)])
def test_many_long_rows(rows, vocab, dtype, parts, top, cap):
    """Eight kinds of rows, each against 64 bits once; all of a kind have its bits."""
    rng = np.random.RandomState(rows + vocab % 1000)
    kinds = logits_of(rng, 8, vocab, dtype)
    kinds[6, vocab // 3:] = -float("inf")
    kinds[7] = torch.from_numpy(rng.randint(0, 300, vocab) / 16.0).to(dtype)
    of = torch.from_numpy(np.concatenate([np.arange(8), rng.randint(0, 8, rows - 8)])).cuda()
    x = kinds.cuda()[of]
    assert (binding.token_logprobs_workspace_bytes(x, top) > 0) == parts
    targets = (of * 1001 % vocab).int()
    got = binding.token_logprobs(x, targets, top, cap)
    logprob, entropy, tops, ids, off, off_entropy = scoring_ref.token_logprobs(kinds.double().numpy(), targets[:8].tolist(), top, cap)
    a = [t[:8].cpu().numpy() for t in got]
    np.testing.assert_array_equal(a[3], ids)
    for have, want, allowed in ((a[0], logprob, off), (a[1], entropy, off_entropy), (a[2], tops, off[:, None])):
        with np.errstate(invalid="ignore"):
            d = np.where(have == want, 0, np.abs(have - want))
        assert (d <= allowed + 2.0 ** -22 * np.abs(np.where(np.isfinite(want), want, 0))).all()
    for t in got:
        assert torch.equal(t.view(torch.int32), t[:8].view(torch.int32)[of])
