"""The oracle of the scoring operators against the other oracles, closed forms and torch in 64 bits (no GPU needed)."""
import math

import numpy as np
import pytest
import torch

from oracle import attention_ref, ref, scoring_ref
from tests.test_gpu_attention_fused import heads


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("kind,asym", [(ref.FP8_E5M2, 1), (ref.E8M0_FLOOR, 0)])
def test_without_masks_it_is_the_fused_attention(causal, kind, asym):
    q, k, v = heads(4, 70, 1, d=64), heads(2, 96, 2, d=64), heads(2, 96, 3, d=64)
    want = attention_ref.fused_attention(q, k, v, 0.125, causal, kind, asym)
    got, allowed = scoring_ref.masked_attention(q, k, v, 0.125, causal, 26, scale_format=kind, asymmetric=asym)
    np.testing.assert_allclose(got.transpose(1, 0, 2), want, rtol=0, atol=2e-6 * np.abs(want).max())
    # what is allowed is BF16's half step and little else: the casts' boundaries are rarely near
    half = 2.0 ** -8 * np.abs(got)
    assert np.median((allowed - half) / np.abs(got).mean()) < 2e-3


def test_a_document_by_itself():
    """Rows of a document that begins at a tile's edge are those of a call of its own; distances do not depend on where it lies."""
    q, k, v = heads(2, 96, 4, d=64), heads(2, 96, 5, d=64), heads(2, 96, 6, d=64)
    first = np.repeat([0, 64], [64, 32])
    how = dict(cap=5.0, slopes=[0.3, 0.01])
    got, _ = scoring_ref.masked_attention(q, k, v, 0.125, first=first, **how)
    alone, _ = scoring_ref.masked_attention(q[:, 64:], k[:, 64:], v[:, 64:], 0.125, **how)
    np.testing.assert_array_equal(got[64:], alone)


def test_ranges():
    lo, hi = scoring_ref.ranges(4, 64, 1, 3, [-5, 2, 9, 0], [1, 2 ** 31 - 1, 63, -1])
    assert lo.tolist() == [0, 2, 9, 0] and hi.tolist() == [1, 4, 5, -1]
    out, allowed = scoring_ref.masked_attention(heads(1, 4, 1, d=64), heads(1, 64, 2, d=64), heads(1, 64, 3, d=64), 0.1, True, 3, [-5, 2, 9, 0], [1, 99, 63, -1])
    assert (out[2:] == 0).all() and (allowed[2:] == 0).all() and (out[:2] != 0).any()


def test_scores():
    s = np.array([-1000.0, -1.0, 0.0, 0.5, 1000.0])
    np.testing.assert_allclose(scoring_ref.score(s, 2.0, 0.25, 4.0), [-3, 2 * math.tanh(-0.5) - 1, -1, 2 * math.tanh(0.25) - 1, 1])


def test_casts_apart():
    p = np.full(32, 0.5)
    p[0] = 1.0  # scale 1/6 -> 0.15625: 0.5 is 3.2 steps of it, far from a boundary
    assert (scoring_ref.cast_between(p, 1e-6, ref.FP8_E5M2, 1) == 0).all()
    p[3] = 2.5 * 0.15625  # between 2 and 3
    d = scoring_ref.cast_between(p, 1e-6, ref.FP8_E5M2, 1)
    assert d[3] == 0.15625 and (np.delete(d, 3) == 0).all()


@pytest.mark.parametrize("cap", [0.0, 7.0])
def test_token_logprobs(cap):
    x = np.random.RandomState(1).randn(5, 300) * 4
    x[1, 5:9] = x[1].max() + 1            # equal ones
    x[2, 100:] = -np.inf
    x[3] = -np.inf
    targets = [7, -1, 299, 2, 300]
    logprob, entropy, tops, ids, off, _ = scoring_ref.token_logprobs(x, targets, 6, cap)
    y = torch.from_numpy(np.where(x > -np.inf, cap * np.tanh(np.where(x > -np.inf, x, 0) / cap) if cap else x, -np.inf))
    z = torch.log_softmax(y, 1)
    assert logprob[1] == logprob[4] == 0 and logprob[2] == -np.inf and logprob[3] == -np.inf
    np.testing.assert_allclose(logprob[0], z[0, 7], rtol=1e-12)
    for r in (0, 1, 2, 4):
        p = z[r].exp()
        np.testing.assert_allclose(entropy[r], -(p[p > 0] * z[r][p > 0]).sum(), rtol=1e-12)
        np.testing.assert_allclose(tops[r], z[r].topk(6).values, rtol=1e-12)
    assert entropy[3] == 0 and (tops[3] == -np.inf).all() and ids[3].tolist() == [0, 1, 2, 3, 4, 5]
    assert ids[1].tolist()[:4] == [5, 6, 7, 8] and (off < 1e-4).all()
