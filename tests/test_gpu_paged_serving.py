"""PagedCache and DecoderLayer.step(): caches that are another layer's, drafts of which rows are taken back."""
import numpy as np
import pytest
import torch

from paper_2411_09909_amd import binding, layer, synth
from tests import gpu_util as G
from tests.test_gpu_paged import FORMATS
from tests.test_gpu_paged_layer import make_layer, ones

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,kv_heads,head_dim", [(8, 1, 64), (8, 4, 64), (4, 1, 128), (4, 2, 128)])
def test_step_refuses_a_cache_of_other_heads(heads, kv_heads, head_dim):
    """Fewer or smaller heads would read keys and values out of the wrong columns of the projection."""
    cfg = layer.LayerConfig(d_model=512, n_heads=8, n_kv_heads=2, head_dim=64, d_ff=1024)
    _, lay = make_layer(cfg, *FORMATS["amxfp4_e5m2"])
    other = layer.LayerConfig(d_model=512, n_heads=heads, n_kv_heads=kv_heads, head_dim=head_dim, d_ff=1024)
    cache = layer.PagedCache(other, lay.fmt, 2, 8, 128, 16)
    before = [t.clone() for t in cache.pools[0]]
    with pytest.raises(binding.AmxError, match="the layer has 2 of 64"):
        lay.step(G.to_dev_bf16(synth.layer_input(2, cfg.d_model, seed=1)), cache, cache.plan(ones(1, 1), 2))
    assert all(torch.equal(a, b) for a, b in zip(before, cache.pools[0]))


def test_rows_of_a_draft_are_taken_back():
    """Drafts of which some rows are accepted, planned a second time from the lengths and the state before: the cache and the layers' outputs are
    bit for bit those of a cache that never saw the drafts, and no page is lost. The accepted rows come into other pages than the draft's
    (two sequences take pages, the first of them for the draft alone); one sequence ends in the same step."""
    cfg = layer.LayerConfig(d_model=512, n_heads=8, n_kv_heads=2, head_dim=64, d_ff=1024)
    layers = [make_layer(cfg, *FORMATS["amxfp4_e5m2"])[1] for _ in range(2)]
    caches = [layer.PagedCache(cfg, layers[0].fmt, 4, 24, 96, 16, layers=2) for _ in range(2)]

    def step(cache, new, x):
        plan = cache.plan(ones(*new), x.shape[0])
        for i, lay in enumerate(layers):
            x = lay.step(x, cache, plan, i)
        return x, plan

    def inputs(rows, seed):
        return G.to_dev_bf16(synth.layer_input(rows, cfg.d_model, seed=seed))

    for cache in caches:
        step(cache, (30, 44, 17, 16), inputs(107, 0))
    other_pages = False
    for n, (draft, accepted) in enumerate([((5, 6, -1, 1), (1, 6, -1, 1)), ((4, 3, 20, 4), (4, 1, 20, 2)), ((3, 4, 1, 20), (0, 2, 1, 11))]):
        rows = inputs(sum(max(v, 0) for v in draft), 10 + n)
        first = np.concatenate([[0], np.cumsum(np.maximum(draft, 0))])
        kept = rows[torch.tensor([first[b] + i for b, a in enumerate(accepted) for i in range(max(a, 0))], device="cuda")]
        tried, plain = caches
        lens, state = tried.lens.clone(), tried.state.clone()
        _, plan = step(tried, draft, rows)
        tried.lens.copy_(lens), tried.state.copy_(state)
        (y, again), (want, expected) = step(tried, accepted, kept), step(plain, accepted, kept)
        assert torch.equal(y, want) and all(torch.equal(a, b) for a, b in zip(again, expected))
        where = torch.cat([plan.slots[first[b]:first[b] + max(a, 0)] for b, a in enumerate(accepted)])
        other_pages |= not torch.equal(where, again.slots)
    assert other_pages
    assert torch.equal(tried.lens, plain.lens) and torch.equal(tried.state, plain.state) and int(plain.state[2]) == 0
    held = [-(-int(v) // 16) for v in plain.lens]
    for b, c in enumerate(held):
        assert torch.equal(tried.table[b, :c], plain.table[b, :c])
    head, count = (int(v) for v in plain.state[:2])
    free = [int(q) for i in range(count) for q in [tried.queue[(head + i) % 24]]]
    assert free == [int(plain.queue[(head + i) % 24]) for i in range(count)]
    assert sorted(free + [int(v) for b, c in enumerate(held) for v in tried.table[b, :c]]) == list(range(24))   # each page once
    slots = torch.cat([tried.table[b, :c].repeat_interleave(16) * 16 + torch.arange(16, device="cuda").repeat(c) for b, c in enumerate(held)])
    slots = torch.cat([slots[16 * sum(held[:b]):][:int(v)] for b, v in enumerate(plain.lens)]).to(torch.int32)
    for p, q in zip(tried.pools, plain.pools):
        for a, b in zip(binding.paged_read(layers[0].fmt, p, slots), binding.paged_read(layers[0].fmt, q, slots)):
            assert torch.equal(a, b)
