"""The oracle of the paged cache against statements that do not need it: pages are never lost or shared, slots name the place that
the table names, the attention is the textbook one over the tokens in order."""
import numpy as np
import pytest

from oracle import paged_ref, ref


def steps(seed, seqs=7, page=16, pages=40, width=6, rows=90, rounds=30):
    rng = np.random.RandomState(seed)
    queue, table = rng.permutation(pages).astype(np.int32), np.full((seqs, width), -1, np.int32)
    lens, state = np.zeros(seqs, np.int32), [rng.randint(pages), pages, 0, 0]
    for _ in range(rounds):
        new = rng.choice([0, 1, 1, 1, 2, 17, 40, -1], seqs)
        yield (lens, new, table, queue, state, page, rows), (out := paged_ref.plan(lens, new, table, queue, state, page, rows))
        lens, state, table, queue = out[0], out[4], out[5], out[6]


@pytest.mark.parametrize("seed", range(5))
def test_pages_are_in_the_queue_or_held_by_one_sequence(seed):
    refused = 0
    for (_, new, _, _, _, page, _), (lens, starts, slots, positions, state, table, queue) in steps(seed):
        pages = len(queue)
        free = [queue[(state[0] + i) % pages] for i in range(state[1])]
        mine = [table[b, j] for b in range(len(lens)) for j in range(-(-lens[b] // page))]
        assert sorted(free + mine) == list(range(pages))
        for b, n in enumerate(new):
            at = range(starts[b], starts[b + 1])
            ok = [positions[t] for t in at if positions[t] >= 0]
            assert ok in ([], list(range(lens[b] - n, lens[b])))
            for t in at:
                if positions[t] >= 0:
                    assert slots[t] == table[b, positions[t] // page] * page + positions[t] % page
        used = slots[slots >= 0]
        assert len(set(used.tolist())) == len(used) and (slots[starts[-1]:] == -1).all()
        refused += state[2]
    assert refused > 0


def test_attention_is_softmax_over_the_tokens_in_order():
    rng = np.random.RandomState(0)
    G, D, page, n = 2, 64, 16, 37
    x = rng.randn(n, 2 * G * D + 4 * D).astype(np.float32)
    pool = {a + b: np.full((5, G) + s, 0x55, np.uint8) for a in "kv" for b, s in (("_codes", (page, D // 2)), ("_scales", (D // 32, page, 2)))}
    table = np.array([[3, 0, 4]])
    slots = table[0][np.arange(n) // page] * page + np.arange(n) % page
    q = paged_ref.write(x, pool, slots, np.arange(n), 4, 10000.0, ref.FP8_E5M2, True)
    q64 = (q.astype(np.uint32) << 16).view(np.float32).astype(np.float64)
    out, weight, _ = paged_ref.attention(q64, pool, table, [n], [0, n], np.arange(n), 0.125, ref.FP8_E5M2, True)
    k, _ = paged_ref.held(pool, "k", table[0], n, ref.FP8_E5M2, True)
    v, _ = paged_ref.held(pool, "v", table[0], n, ref.FP8_E5M2, True)
    want = paged_ref.bf16_from_f32(x[:, 4 * D + G * D:].reshape(n, G, D))
    c, s = ref.quantize(want.reshape(-1, D), 32, ref.FP8_E5M2, True)
    assert np.array_equal(v, ref.dequantize(c, s).reshape(n, G, D))
    for t in (0, 5, n - 1):
        e = np.exp(k[:t + 1, 1] @ q64[t, 3] * 0.125)
        np.testing.assert_allclose(out[t, 3], (e / e.sum()) @ v[:t + 1, 1], rtol=1e-12, atol=1e-12)
    assert np.all(np.abs(out) <= weight + 1e-12)
    none, _, _ = paged_ref.attention(q64, pool, np.array([[-1, 9, 5]]), [n], [0, n], np.arange(n), 0.125, ref.FP8_E5M2, True)
    assert np.all(none == 0)  # no page of the table is in the pool
