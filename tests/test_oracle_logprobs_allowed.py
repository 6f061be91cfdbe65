"""What the oracle allows of log probabilities and entropies is too little for a row that lost a part (no GPU needed)."""
import numpy as np
import pytest

from oracle import scoring_ref


def logits_of(vocab, spread):
    rng = np.random.RandomState(vocab % 1000)
    x = rng.randn(vocab) * spread
    x[rng.randint(0, vocab, 8)] = rng.rand(8) * 16
    return x


@pytest.mark.parametrize("spread", [1.0, 3.0])
@pytest.mark.parametrize("vocab,cut", [(1 << 24, (64, 33)), (130001, (32,)), (50001, (13,)), (33000, (9,)), (9000, (3,)), (20011, (5,))])
@pytest.mark.parametrize("cap", [0.0, 30.0])
def test_a_part_that_is_missing_is_seen(vocab, cut, spread, cap):
    """A part left out of the sum, of the sum of exponentials times distances, or of both."""
    x = logits_of(vocab, spread)
    *_, off, off_entropy = scoring_ref.token_logprobs(x[None], [0], 1, cap)
    y = cap * np.tanh(x / cap) if cap else x
    z = y - y.max()
    e = np.exp(z)
    S, T = e.sum(), (e * z).sum()
    for part, parts in ((at, n) for n in cut for at in (0, n // 2, n - 1)):
        at = slice(part * vocab // parts, (part + 1) * vocab // parts)
        s, t = S - e[at].sum(), T - (e * z)[at].sum()
        entropy = np.log(S) - T / S
        if e[at].sum() < 1e-3 * S or -(e * z)[at].sum() < 1e-3 * S:
            continue  # (a part that hardly counts: spread 3)
        assert abs(np.log(s / S)) > 4 * off[0]
        for missing in ((s, T), (S, t), (s, t)):
            shift = abs(np.log(missing[0]) - missing[1] / missing[0] - entropy)
            # (both missing: what is left may have nearly the entropy of the whole)
            assert shift > off_entropy[0] or (missing == (s, t) and shift < 1e-4 * entropy), (shift, off_entropy[0])


def test_what_is_allowed_stays_small():
    for vocab, most in ((64, 2e-5), (1000, 2e-5), (50001, 1e-4), (130001, 2e-4), (1 << 24, 1e-3)):
        *_, off, off_entropy = scoring_ref.token_logprobs(logits_of(vocab, 1.0)[None], [0], 1, 0.0)
        assert off[0] < most and off_entropy[0] < 16 * most, (vocab, off, off_entropy)


def test_rows_of_one_large_value():
    """Equal values of any size share out the probability: the size of the largest is not part of a difference."""
    for value in (0.0, -3.4e38, 3.4e38, 12345.678):
        logprob, entropy, tops, ids, off, _ = scoring_ref.token_logprobs(np.full((1, 400), value), [7], 3, 0.0)
        np.testing.assert_allclose([logprob[0], *tops[0], -entropy[0]], -np.log(400), rtol=1e-14)
        assert ids[0].tolist() == [0, 1, 2] and off[0] < 1.2e-5
