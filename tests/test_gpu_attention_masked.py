"""Quantized attention whose rows see a range of keys each, with capped scores and biases that fall with distance, against 64 bits.
What may be off is counted in oracle/scoring_ref.py."""
import math

import numpy as np
import pytest
import torch

from oracle import ref, scoring_ref
from paper_2411_09909_amd import binding
from tests import gpu_util as G
from tests.test_gpu_attention_fused import heads
from tests.test_gpu_calls import taken

pytestmark = pytest.mark.gpu
FORMATS = [(ref.FP8_E5M2, 1), (ref.FP8_E5M2, 0), (ref.FP8_E4M3, 1), (ref.E8M0_FLOOR, 1), (ref.E8M0_FLOOR, 0), (ref.E8M0_ROUND, 1)]
FAR = 2 ** 31 - 1


def operands(q, k, v, kind, asym):
    fmt = binding.make_format(kind, asym)
    dev = [G.to_dev_bf16(x.reshape(-1, x.shape[2])).view(x.shape) for x in (q, k, v)]
    return fmt, [t for x, axis in zip(dev, (-1, -1, 1)) for t in binding.quantize_batched(fmt, x, k_axis=axis)]


def ints(v):
    return None if v is None else torch.from_numpy(np.ascontiguousarray(v, np.int32)).cuda()


def slopes_of(H):
    return (2.0 ** (-8.0 * np.arange(1, H + 1) / H)).astype(np.float32)


def check(Hq, Hkv, Sq, Sk, D, kind=ref.FP8_E5M2, asym=1, causal=True, pos0=0, first=None, last=None, cap=0.0, slopes=None, seed=1, rows=None, gain=1.0):
    q, k, v = heads(Hq, Sq, seed, gain, D), heads(Hkv, Sk, seed + 1, d=D), heads(Hkv, Sk, seed + 2, d=D)
    want, allowed = scoring_ref.masked_attention(q, k, v, D ** -0.5, causal, pos0, first, last, cap, slopes, kind, asym, rows)
    fmt, ops = operands(q, k, v, kind, asym)
    need = binding.attention_masked_workspace_bytes(fmt, Hq, Hkv, Sq, Sk, D)
    ws = torch.full((need + 1024,), 0xFF, dtype=torch.uint8, device="cuda")
    out = torch.full((Sq + 2, Hq * D), 7.0, dtype=torch.bfloat16, device="cuda")
    how = dict(causal=causal, pos0=pos0, first=ints(first), last=ints(last), cap=cap, slopes=None if slopes is None else torch.from_numpy(slopes).cuda())
    binding.attention_masked(fmt, *ops, D ** -0.5, **how, out=out[1:-1], workspace=ws[:need])
    assert (out[0] == 7).all() and (out[-1] == 7).all() and (ws[need:] == 0xFF).all()
    got = out[1:-1].float().cpu().numpy().astype(np.float64).reshape(Sq, Hq, D)
    over = np.abs(got - want) / np.maximum(allowed, 1e-300)
    over = over[~np.isnan(want)]
    print("%.3f of what is allowed" % over.max())
    assert np.isfinite(got).all() and over.max() <= 1
    assert torch.equal(binding.attention_masked(fmt, *ops, D ** -0.5, **how), out[1:-1])  # the same bits again, in other buffers
    return got


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kind,asym", FORMATS)
@pytest.mark.parametrize("cap,sloped", [(0.0, False), (20.0, False), (0.0, True), (3.0, True)])
@pytest.mark.parametrize("Sk", [128, 288])  # K and V held whole; brought in by pairs of tiles
def test_formats_and_scores(kind, asym, D, cap, sloped, Sk):
    check(4, 2, 100, Sk, D, kind, asym, cap=cap, pos0=Sk - 110, slopes=slopes_of(4) if sloped else None)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kind,asym", FORMATS)
@pytest.mark.parametrize("cap,sloped", [(0.0, False), (500.0, False), (0.0, True), (500.0, True)])
@pytest.mark.parametrize("Sq,Sk", [(70, 288), (150, 320)])
def test_many_workgroups_walk_tile_by_tile(Sq, Sk, cap, sloped, kind, asym, D):
    """More workgroups than take two tiles to a step; some heads and rows of them against the oracle."""
    H, fmt, at = 534, binding.make_format(kind, asym), [0, 267, 533]
    gen = torch.Generator("cuda").manual_seed(Sq + D)
    q, k, v = (torch.randn((n, s, D), generator=gen, device="cuda").to(torch.bfloat16) for n, s in ((H, Sq), (H // 2, Sk), (H // 2, Sk)))
    ops = [*binding.quantize_batched(fmt, q), *binding.quantize_batched(fmt, k), *binding.quantize_batched(fmt, v, k_axis=1)]
    slopes = torch.rand(H, generator=gen, device="cuda") if sloped else None
    first = torch.randint(-5, Sk - Sq, (Sq,), generator=gen, device="cuda").int()
    out = binding.attention_masked(fmt, *ops, D ** -0.5, pos0=Sk - Sq, first=first, cap=cap, slopes=slopes)
    u16 = lambda x, n: x[n].cpu().view(torch.int16).numpy().view(np.uint16)  # noqa: E731
    of = [h // 2 for h in at]
    want, allowed = scoring_ref.masked_attention(u16(q, at), u16(k, of), u16(v, of), D ** -0.5, True, Sk - Sq, first.cpu().numpy(), None, cap,
                                                 slopes[at].cpu().numpy() if sloped else None, kind, asym, rows := [0, 5, 31, 32, 63, Sq - 1])
    got = out.view(Sq, H, D)[:, at].double().cpu().numpy()
    assert torch.isfinite(out).all() and (np.abs(got - want) <= allowed)[rows].all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kind,asym", [(ref.FP8_E5M2, 1), (ref.E8M0_FLOOR, 0)])
@pytest.mark.parametrize("H,cap,ranged", [(180, 0.0, False), (184, 0.0, True), (304, 20.0, False)])
def test_far_tiles_that_slopes_leave_out(H, cap, ranged, kind, asym, D):
    """Slopes from steep ones, of which the near keys alone count, to none and negative ones; far keys that are large enough to count all the same."""
    Sq, Sk, fmt = 150, 4128, binding.make_format(kind, asym)
    gen = torch.Generator("cuda").manual_seed(H + D)
    q, k, v = (torch.randn((n, s, D), generator=gen, device="cuda").to(torch.bfloat16) for n, s in ((H, Sq), (H // 2, Sk), (H // 2, Sk)))
    k[:, ::97] *= 8
    k[:, 333] *= 60
    ops = [*binding.quantize_batched(fmt, q), *binding.quantize_batched(fmt, k), *binding.quantize_batched(fmt, v, k_axis=1)]
    slopes = torch.exp2(torch.rand(H, generator=gen, device="cuda") * 12 - 9)
    at = [0, 1, 2, 3, H // 2, H - 1]
    slopes[at] = torch.tensor([0.5, 0.1, 0.03, 4.0, 0.0, -0.01], device="cuda")
    last = torch.randint(Sk - Sq - 2000, Sk, (Sq,), generator=gen, device="cuda").int() if ranged else None
    if ranged:
        last[40:80] = -1
    out = binding.attention_masked(fmt, *ops, D ** -0.5, pos0=Sk - Sq, last=last, cap=cap, slopes=slopes)
    u16 = lambda x, n: x[n].cpu().view(torch.int16).numpy().view(np.uint16)  # noqa: E731
    of, n = [h // 2 for h in at], lambda x: None if x is None else x.cpu().numpy()  # noqa: E731
    want, allowed = scoring_ref.masked_attention(u16(q, at), u16(k, of), u16(v, of), D ** -0.5, True, Sk - Sq, None, n(last), cap, n(slopes[at]),
                                                 kind, asym, rows := [0, 31, 77, 128, Sq - 1])
    got = out.view(Sq, H, D)[:, at].double().cpu().numpy()
    assert torch.isfinite(out).all() and (np.abs(got - want) <= allowed)[rows].all()


DOCUMENTS = [1, 2, 31, 32, 1, 33, 64, 5, 40, 7]  # 216 rows


def documents(lengths, prefix=0.0):
    first = np.repeat(np.cumsum([0] + lengths[:-1]), lengths)
    last = np.arange(sum(lengths))
    for at, n in zip(np.cumsum([0] + lengths[:-1]), lengths):
        last[at:at + n] = np.maximum(last[at:at + n], at + int(n * prefix) - 1)
    return first, last


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("cap,sloped", [(0.0, False), (20.0, True)])
@pytest.mark.parametrize("mask", ["documents", "prefixes", "window 1", "window 40", "padding", "some", "any"])
def test_masks(mask, cap, sloped, D):
    rows, causal, rng = 216, True, np.random.RandomState(3)
    first, last = documents(DOCUMENTS, 0.6)
    if mask == "documents":
        last = None
    elif mask == "prefixes":
        causal = False
    elif mask.startswith("window"):
        first, last = np.arange(rows) - int(mask.split()[1]) + 1, None
    elif mask == "padding":
        first, last = None, np.where(np.arange(rows) % 5 < 3, FAR, -1)
    elif mask == "some":  # rows that see nothing, and whole waves and workgroups of them
        last = np.where((np.arange(rows) >= 30) & (np.arange(rows) < 170), -1, np.arange(rows))
        first = None
    else:
        first, last, causal = rng.choice([-2 ** 31, -1, 0, 3, 60, 100, 215, 223, 224, FAR], rows), rng.choice([-2 ** 31, -1, 0, 31, 90, 150, 223, 224, FAR], rows), False
    check(3, 1, rows, 224, D, causal=causal, first=first, last=last, cap=cap, slopes=slopes_of(3) if sloped else None)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv,Sq,Sk,pos0,causal", [(1, 1, 1, 32, 0, True), (1, 1, 1, 32, 31, True), (2, 1, 1, 416, 400, True), (8, 8, 33, 32, 0, True), (5, 5, 129, 96, 7, True),
                                                      (3, 1, 257, 64, 0, False), (16, 2, 40, 352, 300, True), (2, 2, 20, 64, 2 ** 30, True), (4, 4, 128, 160, 32, False)])
def test_shapes(Hq, Hkv, Sq, Sk, pos0, causal, D):
    """One row and key, rows that outnumber the keys, keys behind the last that is seen, positions behind all keys."""
    check(Hq, Hkv, Sq, Sk, D, causal=causal, pos0=pos0, slopes=slopes_of(Hq), cap=30.0)


@pytest.mark.parametrize("D", [64, 128])
def test_large_scores_and_steep_slopes(D):
    check(2, 1, 70, 96, D, gain=40.0, cap=50.0)
    check(2, 1, 70, 96, D, gain=40.0, cap=0.01)
    check(2, 1, 70, 96, D, slopes=np.array([30.0, -0.5], np.float32))
    # far keys only: all scores are shifted alike, by a hundred thousand
    check(2, 1, 3, 1024, D, pos0=10 ** 6, slopes=np.array([0.1, 0.02], np.float32), causal=False)


@pytest.mark.parametrize("D,kind,asym", [(128, ref.FP8_E5M2, 1), (64, ref.E8M0_FLOOR, 1)])
def test_many_tiles(D, kind, asym):
    """Long rows, sampled: a window that crosses workgroups, documents, a long causal row."""
    S, at = 1504, [0, 1, 31, 63, 64, 127, 128, 500, 777, 1023, 1400, 1503]
    check(2, 1, S, S, D, kind, asym, rows=at, cap=30.0, seed=5)
    check(2, 1, S, S, D, kind, asym, rows=at, first=np.arange(S) - 699, slopes=slopes_of(2), seed=6)
    first, last = documents([700, 3, 400, 401], 0.5)
    check(2, 1, S, S, D, kind, asym, rows=at, first=first, last=last, causal=False, seed=7)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kind,asym", FORMATS)
@pytest.mark.parametrize("cap,sloped", [(0.0, False), (20.0, False), (0.0, True), (3.0, True)])
def test_few_rows_are_split_over_the_keys(kind, asym, D, cap, sloped):
    check(2, 1, 5, 1024, D, kind, asym, pos0=1010, cap=cap, slopes=slopes_of(2) if sloped else None)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Sq,Sk,pos0", [(1, 512, 500), (3, 544, 541), (40, 1504, 1460), (130, 768, 600), (33, 4096, 4063)])
@pytest.mark.parametrize("mask", ["causal", "window", "all", "some", "near the end"])
def test_masks_of_split_rows(mask, Sq, Sk, pos0, D):
    """Chunks that no row sees, ranges that end within one, rows that see nothing, a maximum in the first chunk."""
    i, rng = pos0 + np.arange(Sq), np.random.RandomState(Sq)
    how = dict(causal=(mask in ("causal", "window", "near the end")))
    if mask == "window":
        how["first"] = i - 299
    elif mask == "some":
        how["first"], how["last"] = rng.randint(-9, Sk, Sq), np.where(rng.rand(Sq) < 0.3, -1, rng.randint(0, Sk + 9, Sq))
    elif mask == "near the end":
        how["first"] = np.full(Sq, pos0 - 3)
    check(2, 1, Sq, Sk, D, pos0=pos0, cap=30.0, rows=sorted(set(rng.randint(0, Sq, 12).tolist() + [0, Sq - 1])), **how)


def test_scales_that_are_not_finite_stay_where_they_are():
    """Keys that nobody sees may hold any scale; a key's that some rows see spoils those rows alone."""
    Hq, Sq, Sk, D = 2, 96, 160, 128
    fmt, ops = operands(heads(Hq, Sq, 1), heads(1, Sk, 2), heads(1, Sk, 3), ref.FP8_E5M2, 1)
    first, last = np.repeat([0, 40], [40, 56]), np.minimum(np.arange(Sq) + 20, 110)
    how = dict(causal=False, first=ints(first), last=ints(last), cap=20.0)
    want = binding.attention_masked(fmt, *ops, D ** -0.5, **how)
    spoilt = [t.clone() for t in ops]
    spoilt[3][:, 111:] = 0x7F   # K: not a number
    spoilt[5][:, :, 4:] = 0x7C  # V, keys 128 to 159: infinite
    assert torch.equal(binding.attention_masked(fmt, *spoilt, D ** -0.5, **how), want)
    spoilt[3][:, 5] = 0x7F      # seen by rows 0 to 39
    got = binding.attention_masked(fmt, *spoilt, D ** -0.5, **how)
    assert torch.equal(got[40:], want[40:]) and torch.isnan(got[:40].float()).all()


@pytest.mark.parametrize("Sq,Sk", [(320, 320), (20, 1024)])
def test_another_stream_a_graph_and_calls_at_the_same_time(Sq, Sk):
    first = ints(documents([100, 220])[0][:Sq])
    fmt, ops = operands(heads(8, Sq, 1), heads(2, Sk, 2), heads(2, Sk, 3), ref.FP8_E5M2, 1)
    slopes = torch.from_numpy(slopes_of(8)).cuda()
    call = lambda **kw: binding.attention_masked(fmt, *ops, 0.1, pos0=Sk - Sq, first=first, cap=30.0, slopes=slopes, **kw)  # noqa: E731
    want = call()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    torch.cuda.synchronize()
    for s in streams:
        with torch.cuda.stream(s):
            outs.append(call())
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)
    out, ws = torch.zeros_like(want), torch.empty(binding.attention_masked_workspace_bytes(fmt, 8, 2, Sq, Sk, 128), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out=out, workspace=ws)
    for seed in (4, 5):
        ops[0].copy_(operands(heads(8, Sq, seed), heads(2, Sk, 2), heads(2, Sk, 3), ref.FP8_E5M2, 1)[1][0])
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, call())


def test_the_native_way(monkeypatch):
    """With all buffers given the call goes through the native module: the same bits."""
    fmt, ops = operands(heads(4, 70, 1), heads(2, 96, 2), heads(2, 96, 3), ref.FP8_E5M2, 1)
    first, slopes = ints(np.arange(70) - 20), torch.from_numpy(slopes_of(4)).cuda()
    for how in (dict(), dict(first=first, pos0=20), dict(last=first, causal=False, cap=30), dict(first=first, last=first + 9, slopes=slopes, cap=0.0)):
        want = binding.attention_masked(fmt, *ops, 0.1, **how)
        spy = taken(monkeypatch, "attention_masked")
        out = torch.zeros_like(want)
        got = binding.attention_masked(fmt, *ops, 0.1, **how, out=out, workspace=torch.empty(1 << 20, dtype=torch.uint8, device="cuda"))
        assert spy.count == 1 and got is out and torch.equal(want, got)
        monkeypatch.undo()
    out, ws = torch.zeros(70, 512, dtype=torch.bfloat16, device="cuda"), torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    for bad in (dict(first=first[:69]), dict(slopes=slopes[:3]), dict(slopes=slopes.double()), dict(out=out[:69]), dict(workspace=ws[:256]), dict(cap=-1.0)):
        with pytest.raises(binding.AmxError):
            binding.attention_masked(fmt, *ops, 0.1, **{**dict(out=out, workspace=ws), **bad})


def test_wrong_tensors_are_refused():
    fmt, ops = operands(heads(4, 64, 1), heads(2, 64, 2), heads(2, 64, 3), ref.FP8_E5M2, 1)
    call = lambda *o, **kw: binding.attention_masked(fmt, *o, 0.1, **kw)  # noqa: E731
    i = torch.zeros(64, dtype=torch.int32, device="cuda")
    for bad in (dict(first=i[:63]), dict(last=i.long()), dict(first=i.cpu()), dict(slopes=torch.zeros(3, device="cuda")), dict(slopes=torch.zeros(4, device="cuda", dtype=torch.float64)),
                dict(out=torch.zeros(64, 4 * 128, device="cuda")), dict(cap=-1.0), dict(pos0=-1), dict(workspace=torch.zeros(256, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(binding.AmxError):
            call(*ops, **bad)
    with pytest.raises(binding.AmxError):
        call(ops[0], ops[1][..., 0].contiguous(), *ops[2:])  # one scale to a group
    with pytest.raises(binding.AmxError):
        call(*ops[:4], ops[4].transpose(1, 2), ops[5])
    with pytest.raises(binding.AmxError):
        call(ops[0][:3].contiguous(), ops[1][:3].contiguous(), *ops[2:])  # 3 query heads, 2 of keys


def test_the_fused_attention_without_masks():
    """No range, no cap, no slope: the numbers of amxfp4_attention_merged, but for last bits."""
    for D in (64, 128):
        fmt, ops = operands(heads(8, 300, 1, d=D), heads(2, 320, 2, d=D), heads(2, 320, 3, d=D), ref.FP8_E5M2, 1)
        a = binding.attention_masked(fmt, *ops, D ** -0.5, pos0=20).float()
        b = binding.attention(fmt, *ops, D ** -0.5, True, merged=True).float().view_as(a)
        assert (a - b).norm() <= 2.0 ** -9 * b.norm() and math.isfinite(a.sum().item())
