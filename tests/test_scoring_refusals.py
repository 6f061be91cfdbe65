"""What the scoring calls refuse, on the host, before anything is launched (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2411_09909_amd import binding
from tests.test_paged_refusals import BAD_FORMATS, BAD_POOLS, ODD, P, fmt, pool

NOT16 = ctypes.c_void_p(0x1008)
BAD_SCORES = [dict(cap=-1.0), dict(cap=float("nan")), dict(cap=float("inf")), dict(cap=2.0 ** -21), dict(cap=2.0 ** 21), dict(reserved=1),
              dict(slopes=0x1002)]


def scores(cap=0.0, reserved=0, slopes=None):
    return ctypes.byref(binding.AmxScores(cap, reserved, slopes))


@pytest.fixture(scope="module")
def lib():
    return binding.load()


def test_attention_masked(lib):
    def call(f=fmt(), H=8, G=2, Sq=40, Sk=64, D=128, q=(P, P), k=(P, P), v=(P, P), scale=0.1, sc=None, causal=1, pos0=0, first=None, last=None,
             out=P, ws=P, size=1 << 40):
        return lib.amxfp4_attention_masked(None if f is None else ctypes.byref(f), H, G, Sq, Sk, D, *q, *k, *v, scale, sc, causal, pos0, first,
                                           last, out, ws, size, None)
    for f, status in BAD_FORMATS:
        assert call(f) == status
    assert call(None) == -1
    for kw in (dict(H=0), dict(G=0), dict(H=9), dict(H=65536, G=1), dict(Sq=0), dict(Sk=0), dict(Sk=33), dict(Sq=(1 << 20) + 1), dict(Sk=(1 << 20) + 32),
               dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(causal=2), dict(causal=-1), dict(pos0=-1),
               dict(pos0=(1 << 30) + 1), dict(q=(None, P)), dict(q=(P, None)), dict(k=(None, P)), dict(k=(P, None)), dict(v=(None, P)), dict(v=(P, None)),
               dict(out=None), dict(q=(NOT16, P)), dict(k=(NOT16, P)), dict(v=(NOT16, P)), dict(out=NOT16), dict(q=(P, ctypes.c_void_p(0x1001))),
               dict(first=ODD), dict(last=ODD)):
        assert call(**kw) == -1, kw
    for D in (32, 96, 256):
        assert call(D=D) == -2
    for kw in BAD_SCORES:
        assert call(sc=scores(**kw)) == -1, kw
    need = binding.attention_masked_workspace_bytes(fmt(), 8, 2, 40, 64, 128)
    assert need > 0 and binding.attention_masked_workspace_bytes(fmt(), 8, 3, 40, 64, 128) == 0 and binding.attention_masked_workspace_bytes(fmt(), 8, 2, 40, 65, 128) == 0
    few = binding.attention_masked_workspace_bytes(fmt(), 8, 2, 40, 4096, 128)
    assert few > binding.attention_workspace_bytes(fmt(), 8, 2, 40, 4096, 128) and call(Sk=4096, size=few - 1) == -3
    for kw in (dict(ws=None), dict(size=need - 1), dict(ws=ctypes.c_void_p(0x1080))):
        assert call(**kw) == -3, kw
    assert b"workspace" in lib.amxfp4_last_error()


def test_paged_attention_scored(lib):
    f, p = fmt(), pool()

    def call(f=f, p=p, q=P, rows=4, heads=32, table=P, seqs=4, width=4, lens=P, starts=P, positions=P, scale=0.1, sc=scores(cap=30.0), keys=0, out=P,
             ws=P, size=1 << 40):
        return lib.amxfp4_paged_attention_scored(ctypes.byref(f), ctypes.byref(p), q, rows, heads, table, seqs, width, lens, starts, positions,
                                                 scale, sc, keys, out, ws, size, None)
    for bad, status in BAD_FORMATS:
        assert call(f=bad) == status
    for kw, status in BAD_POOLS:
        assert call(p=pool(**kw)) == status
    for kw in BAD_SCORES:
        assert call(sc=scores(**kw)) == -1, kw
    for kw in (dict(q=None), dict(table=None), dict(lens=None), dict(starts=None), dict(positions=None), dict(out=None), dict(rows=0), dict(heads=12),
               dict(seqs=0), dict(seqs=4097), dict(keys=-1), dict(scale=0.0), dict(scale=2.0 ** 101), dict(scale=float("nan")), dict(q=NOT16), dict(lens=ODD)):
        assert call(**kw) == -1, kw
    for kw in (dict(ws=None), dict(size=64), dict(ws=ctypes.c_void_p(0x1080))):
        assert call(**kw) == -3, kw


def test_token_logprobs(lib):
    def call(logits=P, dtype=0, rows=4, vocab=1000, ld=1000, targets=P, cap=0.0, top=5, logprob=P, entropy=P, tops=P, ids=P, ws=P, size=1 << 40):
        return lib.amxfp4_token_logprobs(logits, dtype, rows, vocab, ld, targets, cap, top, logprob, entropy, tops, ids, ws, size, None)
    for kw in (dict(logits=None), dict(dtype=2), dict(dtype=-1), dict(rows=0), dict(rows=-1), dict(rows=(1 << 23) + 1), dict(vocab=0), dict(vocab=(1 << 24) + 1, ld=1 << 25),
               dict(ld=999), dict(ld=(1 << 31) + 1), dict(rows=1 << 20, ld=(1 << 20) + 1), dict(targets=None), dict(logprob=None), dict(tops=None), dict(ids=None),
               dict(top=0), dict(top=-1), dict(top=65), dict(top=5, vocab=4, ld=4), dict(cap=-1.0), dict(cap=float("nan")), dict(cap=2.0 ** 21), dict(cap=2.0 ** -21),
               dict(targets=None, logprob=None, entropy=None, top=0, tops=None, ids=None), dict(logits=ODD), dict(logits=ctypes.c_void_p(0x1001), dtype=1),
               dict(targets=ODD), dict(logprob=ODD), dict(entropy=ODD), dict(tops=ODD), dict(ids=ODD)):
        assert call(**kw) == -1, kw
    big = dict(rows=1, vocab=128000, ld=128000)
    need = lib.amxfp4_token_logprobs_workspace_bytes(0, 1, 128000, 5)
    assert need > 0
    for kw in (dict(ws=None), dict(size=need - 1), dict(ws=ctypes.c_void_p(0x1080))):
        assert call(**big, **kw) == -3, kw
    size = lib.amxfp4_token_logprobs_workspace_bytes
    assert size(0, 1 << 20, 1000, 5) == 0 and size(0, 0, 1000, 5) == 0 and size(2, 1, 128000, 5) == 0 and size(0, 1, 128000, 65) == 0
    assert size(0, 1, 1 << 24, 64) > size(1, 1, 128000, 64) > 0


def test_binding_refuses_host_tensors(lib):
    u = torch.zeros(2, 32, 64, dtype=torch.uint8)
    s = torch.zeros(2, 32, 4, 2, dtype=torch.uint8)
    for call in (lambda: binding.attention_masked(fmt(), u, s, u, s, u, s, 0.1), lambda: binding.token_logprobs(torch.zeros(4, 100))):
        with pytest.raises(binding.AmxError, match="device memory only"):
            call()
