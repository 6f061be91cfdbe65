"""Caps of the scoring calls, which Python settles before the library sees them (no GPU needed)."""
import pytest
import torch

from paper_2411_09909_amd import binding


@pytest.mark.parametrize("cap", [1e-50, -1e-50, 1e-45, 2.0 ** -21, 1e-300, -0.5, 2.0 ** 20 * (1 + 1e-9), 1e300, float("nan"), float("inf")])
def test_caps_that_float32_does_not_hold_are_refused(monkeypatch, cap):
    """A cap that becomes 0 as the library's float32 would be none at all, and one that rounds into range another."""
    monkeypatch.setattr(binding, "_here", lambda *ts: None)
    monkeypatch.setattr(binding, "_need_cuda", lambda *ts: None)
    reached = []

    class Library:
        def __getattr__(self, name):
            return lambda *args: reached.append(name) or 0
    monkeypatch.setattr(binding, "load", lambda: Library())
    monkeypatch.setattr(binding, "_calls", Library())
    monkeypatch.setattr(binding, "_stream", lambda: None)
    fmt, u, s, i = binding.make_format(), torch.zeros(2, 32, 64, dtype=torch.uint8), torch.zeros(2, 32, 4, 2, dtype=torch.uint8), torch.zeros(1, dtype=torch.int32)
    v, vs = torch.zeros(2, 128, 16, dtype=torch.uint8), torch.zeros(2, 128, 1, 2, dtype=torch.uint8)
    pool = (torch.zeros(1, 2, 16, 64, dtype=torch.uint8), torch.zeros(1, 2, 4, 16, 2, dtype=torch.uint8)) * 2
    q, out, ws = torch.zeros(1, 2, 128, dtype=torch.bfloat16), torch.zeros(32, 256, dtype=torch.bfloat16), torch.zeros(4096, dtype=torch.uint8)
    x = torch.zeros(4, 100)
    for given in (dict(), dict(workspace=ws)):
        o = lambda t: {**given, **(dict(out=t) if given else {})}  # noqa: E731
        for call in (lambda: binding.attention_masked(fmt, u, s, u, s, v, vs, 0.1, cap=cap, **o(out)),
                     lambda: binding.paged_attention(fmt, q, pool, i.view(1, 1), i, torch.zeros(2, dtype=torch.int32), i, 0.1, cap=cap, **o(out[:1])),
                     lambda: binding.token_logprobs(x, cap=cap, **o((None, x[:, 0].contiguous(), None, None)))):
            with pytest.raises(binding.AmxError, match="cap"):
                call()
    assert not [n for n in reached if "workspace" not in n]


def test_caps_in_range_and_none():
    assert [binding._cap(c) for c in (None, 0, 0.0, -0.0, 30, 2.0 ** -20, 2 ** 20, torch.tensor(5.0))] == [0, 0, 0, 0, 30, 2.0 ** -20, 2.0 ** 20, 5]
