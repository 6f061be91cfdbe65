"""DecoderLayer.step() over a PagedCache: the calls of the paged cache and the layer's own, run together as a server runs them.

A step is compared in three stages, so that each has a tolerance of its own and a code that a rounding flips early does not hide the
rest: the cache's bytes against the oracle's (bits, from the projection that the layer made), the attention against 64 bits over
those bytes (the roundings counted in test_gpu_paged.allowed), what follows against the oracle's layer from that attention (the bounds
of the whole layer's tests, which count the same operators)."""
import math

import numpy as np
import pytest
import torch

from oracle import layer_ref as L
from oracle import paged_ref
from oracle import ref
from paper_2411_09909_amd import binding, layer, synth
from tests import gpu_util as G
from tests.test_gpu_layer import LAYER_ERR, LAYER_EXACT
from tests.test_gpu_paged import FORMATS, allowed, bits, dev, f64, host_pool

pytestmark = pytest.mark.gpu


def make_layer(cfg, kind, asym, **how):
    w = synth.layer_weights(cfg, seed=0)
    on_gpu = {k: torch.from_numpy(v).cuda() if v.dtype == np.float32 else G.to_dev_bf16(v) for k, v in w.items()}
    return w, layer.DecoderLayer(cfg, on_gpu, binding.make_format(kind, asym), **how)


def ones(*n):
    return torch.tensor(n, dtype=torch.int32, device="cuda")


# (new rows of the four sequences, rows of the batch): prompts of very different lengths; a token each; a chunk among tokens, one
# sequence at its end; rows left over; a new one in the place of the one that ended, another refused (it would need 13 pages)
STEPS = [((150, 3, 0, 40), 193), ((1, 1, 0, 1), 3), ((1, -1, 17, 1), 19), ((1, 0, 1, 2), 9), ((1, 70, 200, 0), 271)]


@pytest.mark.parametrize("name,heads,kv_heads,head_dim,page,how", [
    ("amxfp4_e5m2", 8, 2, 64, 16, {}), ("amxfp4_e5m2", 4, 1, 128, 32, dict(fused_norm=False, fused_glu=False)),
    ("mxfp4_e8m0", 4, 4, 128, 16, dict(prepared_weights=True)), ("amxfp4_e4m3", 16, 2, 64, 16, dict(prepared_weights=True))])
def test_steps_of_a_layer(name, heads, kv_heads, head_dim, page, how):
    kind, asym = FORMATS[name]
    cfg = layer.LayerConfig(d_model=512, n_heads=heads, n_kv_heads=kv_heads, head_dim=head_dim, d_ff=1024)
    w, lay = make_layer(cfg, kind, asym, **how)
    pages = 320 // page + 4
    cache = layer.PagedCache(cfg, lay.fmt, 4, pages, 512, page)
    mirror, table = host_pool(cache.pools[0]), cache.table.cpu().numpy()
    lens, queue, state = np.zeros(4, np.int32), cache.queue.cpu().numpy(), cache.state.cpu().numpy()
    cast = lambda *m: ref.quantize(np.ascontiguousarray(np.concatenate(m, 0)), 32, kind, asym)  # noqa: E731
    after = (cast(w["wo"]), cast(w["wg"], w["wu"]), cast(w["wd"]), kind, asym)
    diff, size, same, refused = 0.0, 0.0, [], []
    for n, (new, rows) in enumerate(STEPS):
        x = synth.layer_input(rows, cfg.d_model, seed=n)
        xd = G.to_dev_bf16(x)
        plan = cache.plan(ones(*new), rows)
        before = [t.clone() for t in cache.pools[0]]
        out = lay.step(xd, cache, plan)

        lens, starts, slots, positions, state, table, queue = paged_ref.plan(lens, new, table, queue, state, page, rows)
        for a, b in zip((*plan, cache.lens, cache.state, cache.table, cache.queue), (lens, starts, slots, positions, state, lens, state, table, queue)):
            np.testing.assert_array_equal(a.cpu().numpy(), b)
        refused.append(int(state[2]))
        # the stages once more, from the pool as it was
        pool = binding.PagedPool(*before)
        proj = lay._qkv(xd)
        q = binding.paged_write(lay.fmt, proj, pool, plan.slots, plan.positions, heads, cfg.rope_theta)
        q_want = paged_ref.write(proj.cpu().numpy(), mirror, slots, positions, heads, cfg.rope_theta, kind, asym)
        seen = positions >= 0
        np.testing.assert_array_equal(bits(q).reshape(q_want.shape)[seen], q_want[seen])
        for a, b, c in zip(mirror.values(), pool, cache.pools[0]):
            np.testing.assert_array_equal(a, c.cpu().numpy())
            assert torch.equal(b, c)
        attn = binding.paged_attention(lay.fmt, q, pool, cache.table, plan.lens, plan.starts, plan.positions, 1 / math.sqrt(head_dim))
        want, weight, bound = paged_ref.attention(f64(bits(q)).reshape(rows, heads, head_dim), mirror, table, lens, starts, positions,
                                                  1 / math.sqrt(head_dim), kind, asym)
        e = np.abs(f64(bits(attn)).reshape(want.shape) - want)[seen]
        assert (e <= allowed(want, weight, bound[..., None], head_dim)[seen]).all()
        assert torch.equal(lay._after_attention(xd, attn)[dev(seen, bool)], out[dev(seen, bool)])
        y = L.f64_from_bf16(L._after_attention(x, bits(attn).reshape(rows, -1), w, cfg, *after))[seen]
        got = L.f64_from_bf16(bits(out).reshape(x.shape))[seen]
        diff, size = diff + ((got - y) ** 2).sum(), size + ((y - L.f64_from_bf16(x)[seen]) ** 2).sum()
        same.append((got == y).ravel())
    print("error %.5f of the update, %.4f of the elements bit-identical" % (math.sqrt(diff / size), np.concatenate(same).mean()))
    assert refused == [0, 0, 0, 0, 1]
    assert math.sqrt(diff / size) <= LAYER_ERR and np.concatenate(same).mean() >= LAYER_EXACT


def test_baseline_layers_share_a_plan_and_a_captured_step_gives_the_eager_bits():
    """Two symmetric layers, one plan to a step: eager, and as a graph that is replayed between other work of the layers (which makes
    their workspace grow)."""
    cfg = layer.LayerConfig(d_model=512, n_heads=4, n_kv_heads=2, head_dim=128, d_ff=1024)
    layers = [make_layer(cfg, ref.E8M0_FLOOR, 0, baseline=True)[1], make_layer(cfg, ref.E8M0_FLOOR, 0, baseline=True)[1]]
    xs = [G.to_dev_bf16(synth.layer_input(3, cfg.d_model, seed=30 + i)) for i in range(6)]

    def start():
        cache = layer.PagedCache(cfg, layers[0].fmt, 3, 60, 1500, 32, layers=2)
        x = G.to_dev_bf16(synth.layer_input(90, cfg.d_model, seed=5))
        plan = cache.plan(ones(60, 1, 29), 90)
        for i, lay in enumerate(layers):
            x = lay.step(x, cache, plan, i)
        return cache

    def step(cache, x, new):
        plan = cache.plan(new, 3)
        for i, lay in enumerate(layers):
            x = lay.step(x, cache, plan, i, max_keys=1000)
        return x

    eager, one = start(), ones(1, 1, 1)
    want = [step(eager, x, one).clone() for x in xs]
    cache, x, new = start(), xs[0].clone(), one.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(start(), x, new)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(cache, x, new)
    for i, (v, y) in enumerate(zip(xs, want)):
        x.copy_(v)
        graph.replay()
        got = out.clone()
        layers[i % 2].forward(G.to_dev_bf16(synth.layer_input(64 * (i + 1), cfg.d_model, seed=i)))
        torch.cuda.synchronize()
        assert torch.equal(got, y)
    for a, b in zip(cache.pools, eager.pools):
        assert all(torch.equal(s, t) for s, t in zip(a, b))
    assert torch.equal(cache.lens, eager.lens) and torch.equal(cache.state, eager.state)


def test_a_prompt_in_one_step_or_in_chunks():
    """The rows of a prompt see the same cache however it is cut: equal bytes, and outputs of a row that do not depend on its batch."""
    cfg = layer.LayerConfig(d_model=512, n_heads=8, n_kv_heads=2, head_dim=64, d_ff=1024)
    _, lay = make_layer(cfg, *FORMATS["amxfp4_e5m2"])
    x = G.to_dev_bf16(synth.layer_input(120, cfg.d_model, seed=1))
    whole = layer.PagedCache(cfg, lay.fmt, 1, 8, 128, 16)
    lay.step(x, whole, whole.plan(ones(120), 120))
    cut = layer.PagedCache(cfg, lay.fmt, 1, 8, 128, 16)
    at = 0
    for n in (64, 1, 31, 24):
        lay.step(x[at:at + n], cut, cut.plan(ones(n), n))
        at += n
    torch.cuda.synchronize()
    assert int(cut.lens) == 120
    # (the projection's kernel, and with it the order of its FP32 sums, goes with the number of rows: a BF16 value that lies within
    # 2^-20 of a rounding boundary, some 2^-11 of them, can be a step off, and with it a code, by at most 2 of 6 of the group's largest,
    # or the scale, by a quarter: 1 / 4 + 5 / 4 / 3 = 0.67. A scale takes 32 values along: at most 2 % of them differ)
    slots = torch.arange(120, dtype=torch.int32, device="cuda")
    for a, b in zip(binding.paged_read(lay.fmt, whole.pools[0], slots), binding.paged_read(lay.fmt, cut.pools[0], slots)):
        big = a.float().view(120, -1, 32).abs().amax(-1, keepdim=True)
        assert ((a.float() - b.float()).view(120, -1, 32).abs() <= 0.67 * big).all()
        assert (a == b).float().mean() > 0.98


def test_step_refuses_a_cache_of_another_kind():
    cfg = layer.LayerConfig(d_model=512, n_heads=8, n_kv_heads=2, head_dim=64, d_ff=1024)
    _, lay = make_layer(cfg, *FORMATS["amxfp4_e5m2"])
    x = G.to_dev_bf16(synth.layer_input(2, cfg.d_model, seed=1))
    good = layer.PagedCache(cfg, lay.fmt, 2, 8, 128, 16)
    plan = good.plan(ones(1, 1), 2)
    symmetric = layer.PagedCache(cfg, binding.make_format(ref.FP8_E5M2, 0), 2, 8, 128, 16)
    with pytest.raises(binding.AmxError, match="scales"):
        lay.step(x, symmetric, plan)
    with pytest.raises(binding.AmxError):
        lay.step(x[:1], good, plan)   # one row, a plan for two
    with pytest.raises(binding.AmxError):
        good.plan(ones(1, 1, 1), 2)
    lay.step(x, good, plan)
    torch.cuda.synchronize()
