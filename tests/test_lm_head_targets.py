"""Targets of LMHead.logprobs(), checked before the rows are cut into parts (no GPU needed)."""
import pytest
import torch

from paper_2411_09909_amd import binding, layer


def head_of(at_once):
    head = layer.LMHead.__new__(layer.LMHead)  # (no weights: nothing is multiplied)
    head.cap, head.rows_at_once = 0.0, at_once
    return head


@pytest.mark.parametrize("rows,at_once", [(64, 32), (64, 64), (70, 32), (3, 1024)])
@pytest.mark.parametrize("more", [-1, 1, 32])
def test_targets_go_with_the_rows(monkeypatch, rows, at_once, more):
    head, said = head_of(at_once), []
    monkeypatch.setattr(head, "logits", lambda x: x, raising=False)
    monkeypatch.setattr(binding, "token_logprobs", lambda *args, **how: said.append(args))
    x = torch.zeros(rows, 8)
    if rows + more >= 0:
        with pytest.raises(binding.AmxError, match="of %d" % rows):
            head.logprobs(x, torch.zeros(rows + more, dtype=torch.int32))
    for bad in (torch.zeros(rows), torch.zeros(rows, dtype=torch.int64), torch.zeros(rows, 1, dtype=torch.int32)):
        with pytest.raises(binding.AmxError):
            head.logprobs(x, bad)
    assert not said
    head.logprobs(x, torch.zeros(rows, dtype=torch.int32))
    head.logprobs(x)
    assert len(said) == 2 * -(-rows // at_once)
