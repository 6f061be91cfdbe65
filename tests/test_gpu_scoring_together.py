"""Scoring text as a program does it: documents packed into one pass through layers with capped scores and distance biases, the log
probabilities of their tokens, and single tokens that continue them over the paged cache."""
import math

import numpy as np
import pytest
import torch

from oracle import scoring_ref
from paper_2411_09909_amd import binding, layer
from tests.test_gpu_attention_masked import ints, slopes_of
from tests.test_gpu_paged import FORMATS, bits
from tests.test_gpu_paged_layer import make_layer, ones
from tests.test_gpu_token_logprobs import check as check_logprobs

pytestmark = pytest.mark.gpu


def config(**how):
    return layer.LayerConfig(**{**dict(d_model=512, n_heads=8, n_kv_heads=2, head_dim=64, d_ff=1024), **how})


def u16(t):
    return bits(t).reshape(t.shape)


@pytest.mark.parametrize("name,how", [("amxfp4_e5m2", dict(score_cap=20.0)), ("mxfp4_e8m0", dict(n_heads=4, n_kv_heads=4, head_dim=128)),
                                      ("amxfp4_e4m3", dict(n_heads=4, n_kv_heads=1, head_dim=128, score_cap=5.0))])
@pytest.mark.parametrize("prefixes", [False, True])
def test_packed_documents_through_a_layer(name, how, prefixes):
    kind, asym = FORMATS[name]
    cfg = config(**how)
    H, G, D, S = cfg.n_heads, cfg.n_kv_heads, cfg.head_dim, 160
    slopes = slopes_of(H)
    _, lay = make_layer(cfg, kind, asym, fused_attention=True, slopes=torch.from_numpy(slopes).cuda())
    x = torch.randn(S, cfg.d_model, device="cuda").to(torch.bfloat16)
    first = np.repeat([0, 50, 83], [50, 33, S - 83])
    last = np.arange(S)
    last[50:70] = 69  # a prefix of 20 rows
    last[150:] = -1   # rows without text
    masks = dict(first=ints(first), **(dict(last=ints(last)) if prefixes else {}))
    out = lay.forward(x, **masks)
    # the stages once more: what the layer makes of the attention over its own queries, keys and values
    qkv = lay._qkv(x)
    q, k = (binding.split_heads_rope(qkv, col, n, D, True, 0, cfg.rope_theta) for col, n in ((0, H), (H * D, G)))
    v = binding.split_heads_rope(qkv, (H + G) * D, G, D, False)
    cast = lambda y, axis=-1: binding.quantize_batched(lay.fmt, y, k_axis=axis)  # noqa: E731
    attn = binding.attention_masked(lay.fmt, *cast(q), *cast(k), *cast(v, 1), 1 / math.sqrt(D), causal=not prefixes, cap=cfg.score_cap, slopes=lay.slopes,
                                    **masks)
    assert torch.equal(lay._after_attention(x, attn), out)
    want, allowed = scoring_ref.masked_attention(u16(q), u16(k), u16(v), 1 / math.sqrt(D), not prefixes, 0, first, last if prefixes else None, cfg.score_cap,
                                                 slopes, kind, asym)
    assert (np.abs(attn.double().cpu().numpy().reshape(want.shape) - want) <= allowed).all()
    if prefixes:
        assert not attn[150:].any()


def test_a_layer_without_fused_attention_refuses_masks():
    cfg = config(score_cap=10.0)
    _, lay = make_layer(cfg, binding.FP8_E5M2, True)
    x = torch.randn(32, cfg.d_model, device="cuda").to(torch.bfloat16)
    with pytest.raises(binding.AmxError, match="fused_attention"):
        lay.forward(x)
    _, lay = make_layer(config(), binding.FP8_E5M2, True)
    with pytest.raises(binding.AmxError, match="fused_attention"):
        lay.forward(x, first=torch.zeros(32, dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("vocab,rows,at_once", [(1001, 70, 32), (4096, 96, 1024)])
def test_log_probabilities_behind_a_head(vocab, rows, at_once):
    fmt = binding.make_format()
    gen = torch.Generator("cuda").manual_seed(vocab)
    weight = (torch.randn(vocab, 512, generator=gen, device="cuda") * 0.1).to(torch.bfloat16)
    x = torch.randn(rows, 512, generator=gen, device="cuda").to(torch.bfloat16)
    head = layer.LMHead(weight, torch.ones(512, device="cuda"), fmt, cap=30.0, rows_at_once=at_once)
    targets = torch.randint(-1, vocab, (rows,), generator=gen, device="cuda").int()
    got = head.logprobs(x, targets, top=5)
    logits = torch.cat([head.logits(x[i:i + at_once]) for i in range(0, rows, at_once)])
    check_logprobs(logits.cpu(), targets.tolist(), 5, 30.0)
    for a, b in zip(got, binding.token_logprobs(logits, targets, 5, 30.0)):
        assert torch.equal(a, b)
    assert head.logprobs(x).logprobs is None and torch.equal(head.logprobs(x).entropy, got.entropy)


def test_texts_are_scored_and_continued():
    """A greedy step over the cache behind a scored prompt: layers with capped scores and slopes, eager and as a graph."""
    cfg = config(score_cap=15.0)
    slopes = torch.from_numpy(slopes_of(cfg.n_heads)).cuda()
    layers = [make_layer(cfg, binding.FP8_E5M2, True, slopes=slopes)[1] for _ in range(2)]
    fmt = layers[0].fmt
    gen = torch.Generator("cuda").manual_seed(3)
    weight = (torch.randn(1000, cfg.d_model, generator=gen, device="cuda") * 0.1).to(torch.bfloat16)
    embed = torch.randn(1000, cfg.d_model, generator=gen, device="cuda").to(torch.bfloat16)
    head = layer.LMHead(weight, torch.ones(cfg.d_model, device="cuda"), fmt, cap=30.0)
    prompts = [torch.randint(0, 1000, (n,), generator=gen, device="cuda") for n in (33, 7, 64)]

    def step(cache, tokens, rows):
        plan = cache.plan(rows, len(tokens))
        x = embed[tokens]
        for i, lay in enumerate(layers):
            x = lay.step(x, cache, plan, i)
        return x

    def run(how):
        cache = layer.PagedCache(cfg, fmt, 3, 30, 512, 16, layers=2)
        x = step(cache, torch.cat(prompts), ones(*map(len, prompts)))
        scores = head.logprobs(x[:-1], torch.cat(prompts).int()[1:], top=1)
        ends = torch.tensor([32, 39, 103], device="cuda")
        token = head.logprobs(x[ends], top=1).top_ids[:, 0].long()
        said, each = [token.clone()], ones(1, 1, 1)
        graph = None
        for _ in range(3):
            if how == "graph" and graph is None and len(said) == 2:
                graph = torch.cuda.CUDAGraph()
                before = [t.clone() for t in (cache._now, cache.queue, cache.table)]
                with torch.cuda.graph(graph):
                    after = head.logprobs(step(cache, token, each), top=3)
                for t, b in zip((cache._now, cache.queue, cache.table), before):
                    t.copy_(b)
            if graph is not None:
                graph.replay()
            else:
                after = head.logprobs(step(cache, token, each), top=3)
            torch.cuda.synchronize()
            token.copy_(after.top_ids[:, 0])
            said.append(token.clone())
        return scores, torch.stack(said), after

    a, b = run("eager"), run("graph")
    assert torch.isfinite(a[0].logprobs).all() and (a[0].logprobs <= 0).all() and (a[0].logprobs <= a[0].top_logprobs[:, 0]).all()
    assert torch.equal(a[1], b[1]) and all(torch.equal(x, y) for x, y in zip(a[2][1:], b[2][1:]))
