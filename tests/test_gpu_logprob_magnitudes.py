"""Logits of any finite size: tokens that a program rules out with its type's lowest value, and sizes whose differences leave FP32's range."""
import numpy as np
import pytest
import torch

from oracle import scoring_ref
from tests.test_gpu_token_logprobs import logits_of, run

pytestmark = pytest.mark.gpu


def check(x, targets, top, cap=0.0):
    """As test_gpu_token_logprobs.check(); log probabilities below FP32's range are -inf."""
    got = run(x, targets, top, cap)
    logprob, entropy, tops, ids, off, off_entropy = scoring_ref.token_logprobs(x.double().cpu().numpy(), targets, top, cap)
    np.testing.assert_array_equal(got[3], ids)
    for a, b, allowed in ((got[0], logprob, off), (got[1], entropy, off_entropy), (got[2], tops, off[:, None])):
        with np.errstate(over="ignore", invalid="ignore"):
            b = np.where(np.abs(b) > 2.0 ** 128 - 2.0 ** 103, -np.inf, b)
            d = np.where(a == b, 0, np.abs(a - b))
            assert (d <= allowed + 2.0 ** -22 * np.abs(np.where(np.isfinite(b), b, 0)) + 2.0 ** -100).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [70, 2999, 33000, 128000])
@pytest.mark.parametrize("cap", [0.0, 30.0])
def test_tokens_ruled_out_by_the_lowest_value(vocab, cap, dtype):
    rng = np.random.RandomState(vocab)
    lowest = torch.finfo(dtype).min
    x = logits_of(rng, 7, vocab, dtype)
    x[0, 5:] = lowest
    x[1] = lowest
    x[2, :-1] = lowest
    x[3, rng.rand(vocab) < 0.9] = lowest
    x[4, vocab // 3:] = lowest
    x[5, ::2] = lowest
    x[6, :vocab // 2] = lowest
    x[6, 3] = -float("inf")
    targets = [0, 3, vocab - 1, 0, 1, vocab - 1, vocab - 2]
    for top in (5, 20, 64):
        check(x, targets, top, cap)
    for row in (0, 1, 4, 6):
        check(x[row:row + 1], targets[row:row + 1], 20, cap)
    check(x, [7, 9, 0, 4, vocab - 1, 2, 0], 3, cap)  # targets that are ruled out


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [12, 3000, 60000])
def test_logits_of_the_largest_sizes(vocab, dtype):
    rng = np.random.RandomState(vocab)
    x = logits_of(rng, 6, vocab, dtype)
    most = torch.finfo(dtype).max
    x[0, 3], x[0, 7] = 2.0 ** 127, -2.0 ** 127
    x[1, 3], x[1, 7] = most, -most
    x[2] = -most
    x[2, 5] = most
    x[3] = most
    x[3, ::2] = -most
    x[4, vocab - 1] = -most
    x[5] = 0
    x[5, :5] = torch.tensor([2.0 ** 126, 2.0 ** 126, -2.0 ** 127, -2.0 ** 120, 2.0 ** 126], dtype=dtype)
    for targets in ([3, 3, 5, 1, 0, 0], [7, 7, 1, 2, vocab - 1, 2], [-1] * 6):
        check(x, targets, 6)
        check(x, targets, 6, cap=50.0)
    for row in range(6):
        check(x[row:row + 1], [3], 12)
