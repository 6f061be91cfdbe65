"""Log probabilities of tokens, entropy and top alternatives against 64 bits. What may be off is counted in oracle/scoring_ref.py."""
import numpy as np
import pytest
import torch

from oracle import scoring_ref
from paper_2411_09909_amd import binding
from tests.test_gpu_calls import taken

pytestmark = pytest.mark.gpu
INF = float("inf")


def logits_of(rng, rows, vocab, dtype, spread=3.0):
    x = rng.randn(rows, vocab) * spread
    at = rng.randint(0, vocab, (rows, 8))
    x[np.arange(rows)[:, None], at] = rng.rand(rows, 8) * 16
    return torch.from_numpy(x.astype(np.float32)).to(dtype)


def run(x, targets, top, cap, ld=None, before=0):
    """The call on rows of x that lie `ld` apart in a wider buffer of NaN, `before` elements behind its beginning."""
    rows, vocab = x.shape
    ld = ld or vocab
    flat = torch.full((before + rows * ld + 8,), float("nan"), dtype=x.dtype, device="cuda")
    view = flat[before:before + rows * ld].view(rows, ld)[:, :vocab]
    view.copy_(x)
    t = None if targets is None else torch.tensor(targets, dtype=torch.int32, device="cuda")
    f = lambda *shape: torch.full(shape, 77.0, device="cuda")  # noqa: E731
    guarded = [f(rows + 2), f(rows + 2), f(rows + 2, top), torch.full((rows + 2, top), 77, dtype=torch.int32, device="cuda")]
    out = [g[1:-1] for g in guarded]
    if targets is None:
        out[0] = None
    if not top:
        out[2] = out[3] = None
    need = binding.token_logprobs_workspace_bytes(view, top)
    ws = torch.full((need + 512,), 0xFF, dtype=torch.uint8, device="cuda")
    got = binding.token_logprobs(view, t, top, cap, out=out, workspace=ws[:max(need, 256)])
    assert all((g[0] == 77).all() and (g[-1] == 77).all() for g in guarded) and (need == 0 or (ws[need:] == 0xFF).all())
    again = binding.token_logprobs(view, t, top, cap)
    for a, b in zip(got, again):
        assert (a is None) == (b is None) and (a is None or torch.equal(a.view(torch.int32), b.view(torch.int32)))
    return [None if a is None else a.cpu().numpy() for a in got]


def check(x, targets, top, cap=0.0, **how):
    got = run(x, targets, top, cap, **how)
    logprob, entropy, tops, ids, off, off_entropy = scoring_ref.token_logprobs(x.double().cpu().numpy(), targets, top, cap)

    def near(a, b, allowed):
        with np.errstate(invalid="ignore"):
            d = np.where(a == b, 0, np.abs(a - b))
        over = d / (allowed + 2.0 ** -22 * np.abs(np.where(np.isfinite(b), b, 0)) + 2.0 ** -100)
        assert over.max() <= 1, over.max()
        return float(over.max())
    worst = [near(got[1], entropy, off_entropy)]
    if targets is not None:
        worst.append(near(got[0], logprob, off))
    if top:
        np.testing.assert_array_equal(got[3], ids)
        worst.append(near(got[2], tops, off[:, None]))
    print("%.3f of what is allowed" % max(worst))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [1, 2, 3, 5, 31, 64, 65, 257, 1000, 1023, 1024, 1025, 2048, 4099, 20011, 50001, 130001])
@pytest.mark.parametrize("cap", [0.0, 30.0])
def test_vocabularies(vocab, dtype, cap):
    rng = np.random.RandomState(vocab)
    rows = 3
    check(logits_of(rng, rows, vocab, dtype), [0, vocab - 1, vocab // 2], min(vocab, 20), cap)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("top", [0, 1, 2, 5, 20, 63, 64])
@pytest.mark.parametrize("rows,vocab", [(1, 64), (1, 1500), (2, 33000), (70, 9000), (2100, 300)])
def test_alternatives(rows, vocab, top, dtype):
    rng = np.random.RandomState(rows + top)
    check(logits_of(rng, rows, vocab, dtype), rng.randint(0, vocab, rows).tolist(), top)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("before,ld", [(1, 5003), (2, 5001), (3, 5002), (4, 5008), (5, 5005), (7, 5004), (0, 6000), (6, 5001)])
def test_rows_that_begin_anywhere(before, ld, dtype):
    rng = np.random.RandomState(ld + before)
    check(logits_of(rng, 9, 5001, dtype), rng.randint(0, 5001, 9).tolist(), 7, before=before, ld=ld)
    check(logits_of(rng, 9, 3, dtype), [0, 1, 2] * 3, 3, before=before, ld=ld % 13 + 3)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,vocab", [(3, 700), (1, 40000), (2100, 2500)])
def test_equal_logits_go_by_id(rows, vocab, dtype):
    """All equal, equal in steps, ascending, descending, zeros of both signs: more elements reach the bound than are put in order at once."""
    rng = np.random.RandomState(vocab)
    for x in (np.zeros((rows, vocab)), rng.randint(0, 4, (rows, vocab)), rng.randint(0, 300, (rows, vocab)) / 16, np.tile(np.arange(vocab) // 3, (rows, 1)) * 2.0 ** -6,
              np.tile(-np.arange(vocab) // 3, (rows, 1)) * 2.0 ** -6, np.where(rng.rand(rows, vocab) < 0.5, 0.0, -0.0)):
        for top in (1, 20, 64):
            check(torch.from_numpy(x.astype(np.float32)).to(dtype), rng.randint(0, vocab, rows).tolist(), top)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [70, 3000, 33000])
def test_tokens_ruled_out(vocab, dtype):
    rng = np.random.RandomState(vocab)
    x = logits_of(rng, 8, vocab, dtype)
    x[0, 5:] = -INF                     # fewer are left than are asked for
    x[1] = -INF
    x[2, :-1] = -INF                    # one is left
    x[3, rng.rand(vocab) < 0.9] = -INF
    x[4, 40:] = -INF
    x[5] = -INF
    x[6, ::2] = -INF
    for cap in (0.0, 5.0):
        check(x, [0, 3, vocab - 1, 0, vocab - 1, -1, 0, 1], 20, cap)
        check(x, [9, vocab, vocab - 2, -2 ** 31, 2 ** 31 - 1, -1, 5, 1], 0, cap)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [70, 2999, 33000, 128000])
def test_tokens_whole_parts_ruled_out(vocab, dtype):
    rng = np.random.RandomState(vocab + 1)
    x = logits_of(rng, 6, vocab, dtype)
    x[0, vocab // 3:] = -INF
    x[1, :vocab // 2] = -INF
    x[2] = -INF
    x[3, 40:] = -INF
    x[4, :-30] = -INF
    x[5, rng.rand(vocab) < 0.999] = -INF
    for top in (20, 64):
        check(x, [0, vocab - 1, 5, 39, vocab - 1, 0], top)
        for row in range(6):            # (one row alone is in parts)
            check(x[row:row + 1], [1], top, 5.0 * (row % 2))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [30, 2000, 60000])
def test_what_is_not_a_number(vocab, dtype):
    rng = np.random.RandomState(vocab)
    x = logits_of(rng, 5, vocab, dtype)
    good = x.clone()
    x[0, 7], x[1, vocab - 1], x[2], x[4, 3] = float("nan"), INF, float("nan"), -INF
    good[4, 3] = -INF
    targets = [1, 1, 1, 1, -1]
    for cap in (0.0, 30.0):
        got, want = run(x, targets, 12, cap), run(good, targets, 12, cap)
        spoilt = [0, 2] if cap else [0, 1, 2]  # (a capped +inf is the cap)
        for a, b in zip(got, want):
            np.testing.assert_array_equal(a[3:], b[3:])
        assert all(np.isnan(a[spoilt]).all() for a in got[:3])
        assert ((got[3] >= -1) & (got[3] < vocab)).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_large_and_small_logits(dtype):
    rng = np.random.RandomState(7)
    x = logits_of(rng, 6, 3000, torch.float32)
    x[0] *= 1000
    x[1] = x[1] * 1e-6
    x[2] = x[2] * 10 + 5000
    x[3] = x[3] - 1e6
    x[4, 17], x[4, 18] = 1e37, -1e37
    x = x.to(dtype)
    check(x, [3, 4, 5, 6, 17, 8], 10)
    check(x, [3, 4, 5, 6, 18, 8], 10, cap=50.0)
    check(x, [3, 4, 5, 6, 18, 8], 10, cap=2.0 ** -20)


def test_the_largest_vocabulary_and_many_rows():
    rng = np.random.RandomState(2)
    check(logits_of(rng, 1, 1 << 24, torch.bfloat16, spread=1.0), [12345678], 64)
    x = logits_of(rng, 1, 997, torch.float32).repeat(30000, 1)
    x[:, 0] = torch.arange(30000) % 50 / 8
    got = binding.token_logprobs(x.cuda(), torch.zeros(30000, dtype=torch.int32, device="cuda"), 3)
    want = scoring_ref.token_logprobs(x[:50].double().numpy(), [0] * 50, 3, 0.0)
    for a, b in zip(got[:3], want):
        np.testing.assert_allclose(a.cpu().numpy().reshape((600, 50) + b.shape[1:]), np.broadcast_to(b, (600, 50) + b.shape[1:]), rtol=0, atol=1e-5)
    assert (got[3].cpu().numpy().reshape(600, 50, 3) == want[3]).all()


def test_another_stream_and_a_graph():
    rng = np.random.RandomState(4)
    x = logits_of(rng, 5, 50000, torch.float32).cuda()
    t = torch.tensor([1, 2, 3, 4, 5], dtype=torch.int32, device="cuda")
    want = binding.token_logprobs(x, t, 10)
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        other = binding.token_logprobs(x, t, 10)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, other))
    out = binding.TokenLogprobs(*(torch.zeros_like(a) for a in want))
    ws = torch.empty(binding.token_logprobs_workspace_bytes(x, 10), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.token_logprobs(x, t, 10, out=out, workspace=ws)
    for seed in (1, 2, 3):
        x.copy_(logits_of(np.random.RandomState(seed), 5, 50000, torch.float32))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(binding.token_logprobs(x, t, 10), out))


def test_the_native_way(monkeypatch):
    """With all buffers given the calls go through the native module; what it does not take is refused as before."""
    x, t = torch.randn(3, 700, device="cuda"), torch.tensor([1, 2, 700], dtype=torch.int32, device="cuda")
    want = binding.token_logprobs(x, t, 4, 30.0)
    for targets, top, drop in ((t, 4, ()), (None, 4, (0,)), (t, 0, (2, 3)), (t, 4, (1,))):
        spy = taken(monkeypatch, "token_logprobs")
        out = tuple(None if i in drop else torch.zeros_like(a) for i, a in enumerate(want))
        got = binding.token_logprobs(x, targets, top, 30, out=out, workspace=torch.empty(1 << 20, dtype=torch.uint8, device="cuda"))
        assert spy.count == 1 and all(b is None or torch.equal(a, b) for a, b in zip(want, got))
        monkeypatch.undo()
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    good = [torch.zeros_like(a) for a in want]
    for i, bad in ((0, good[0][:2]), (1, good[1].double()), (2, good[2][:, :3]), (3, good[3].float()), (2, good[2].cpu())):
        with pytest.raises(binding.AmxError):
            binding.token_logprobs(x, t, 4, out=[bad if j == i else a for j, a in enumerate(good)], workspace=ws)
    with pytest.raises(binding.AmxError):
        binding.token_logprobs(torch.randn(1, 200000, device="cuda"), out=(None, good[1][:1], None, None), workspace=ws[:256])  # too small


def test_wrong_tensors_are_refused():
    x, t = torch.zeros(4, 100, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    for bad in (lambda: binding.token_logprobs(x.half(), t), lambda: binding.token_logprobs(x.t(), t), lambda: binding.token_logprobs(x, t.long()),
                lambda: binding.token_logprobs(x, t[:3]), lambda: binding.token_logprobs(x, t, 65), lambda: binding.token_logprobs(x[:, :5], t, 6),
                lambda: binding.token_logprobs(x, t, 2, out=(x[:, 0].contiguous(), x[0, :4], x[:, :2].contiguous(), t)), lambda: binding.token_logprobs(x, t, cap=-1.0),
                lambda: binding.token_logprobs(x[:1].expand(4, 100), t)):
        with pytest.raises(binding.AmxError):
            bad()
