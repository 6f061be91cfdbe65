"""The paged key / value cache on the GPU: bookkeeping and stored bytes exactly as the oracle has them, the attention within what
its roundings allow, the three together as a serving step uses them."""
import math

import numpy as np
import pytest
import torch

from oracle import paged_ref, ref
from paper_2411_09909_amd import binding

pytestmark = pytest.mark.gpu
THETA = 500000.0
FORMATS = {"amxfp4_e5m2": (binding.FP8_E5M2, True), "mxfp4_e5m2": (binding.FP8_E5M2, False), "amxfp4_e4m3": (binding.FP8_E4M3, True),
           "mxfp4_e4m3": (binding.FP8_E4M3, False), "amxfp4_e8m0": (binding.E8M0_FLOOR, True), "mxfp4_e8m0": (binding.E8M0_FLOOR, False),
           "amxfp4_round": (binding.E8M0_ROUND, True), "mxfp4_round": (binding.E8M0_ROUND, False)}
NAMES = ("k_codes", "k_scales", "v_codes", "v_scales")


def dev(a, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(a, dtype)).cuda()


def bits(t):
    return t.cpu().contiguous().view(torch.int16).numpy().view(np.uint16)


def f64(b):
    return (b.astype(np.uint32) << 16).view(np.float32).astype(np.float64)


# ---- plan -----------------------------------------------------------------------------------------------------------

def run_plan(lens, new, table, queue, state, page, rows):
    t, q = dev(table), dev(queue)
    out = [torch.full((n,), 77, dtype=torch.int32, device="cuda") for n in (len(lens), len(lens) + 1, rows, rows, 4)]
    plan = binding.paged_plan(dev(lens), dev(new), t, q, dev(state), page, out=out)
    again = binding.paged_plan(dev(lens), dev(new), t, q, dev(state), page, rows=rows)  # the same once more changes nothing
    assert all(torch.equal(a, b) for a, b in zip(plan, again))
    return [v.cpu().numpy() for v in plan] + [t.cpu().numpy(), q.cpu().numpy()]


def check_plan(*args):
    got, want = run_plan(*args), paged_ref.plan(*args)
    for name, a, b in zip(("lens", "starts", "slots", "positions", "state", "table", "queue"), got, want):
        np.testing.assert_array_equal(a, b, err_msg=name)
    return want


@pytest.mark.parametrize("seqs,page,pages,width,rows,chunk", [
    (1, 16, 1, 1, 1, 1), (1, 64, 9, 8, 700, 500), (5, 32, 40, 6, 64, 40), (64, 64, 300, 20, 64, 1), (255, 16, 900, 8, 400, 3),
    (256, 16, 900, 8, 300, 3), (257, 128, 700, 4, 5000, 60), (1000, 16, 3000, 50, 9000, 20), (4096, 16, 9000, 4, 5000, 2),
    (300, 16, 150, 6, 500, 9)])
def test_plan_over_many_steps(seqs, page, pages, width, rows, chunk):
    rng = np.random.RandomState(seqs)
    lens, table = np.zeros(seqs, np.int32), np.full((seqs, width), -1, np.int32)
    queue, state = rng.permutation(pages).astype(np.int32), [rng.randint(pages), pages, 0, 0]
    for _ in range(12):
        new = rng.choice([0, 1, 1, 1, rng.randint(1, chunk + 1), -1], seqs)
        out = check_plan(lens, new, table, queue, state, page, rows)
        lens, state, table, queue = out[0], out[4], out[5], out[6]


def test_plan_of_nothing_and_of_everything_refused():
    table, queue = np.full((3, 4), -1), np.arange(8)
    check_plan([0, 0, 0], [0, 0, 0], table, queue, [3, 8, 0, 0], 16, 5)
    check_plan([0, 0, 0], [1, 1, 1], table, queue, [3, 0, 0, 0], 16, 5)      # no free page
    check_plan([0, 0, 0], [65, 64, 1], table, queue, [7, 8, 0, 0], 16, 200)   # one too long for its row of the table
    check_plan([0, 0, 0], [3, 3, 3], table, queue, [7, 8, 0, 0], 16, 7)       # the last does not fit the batch
    check_plan([0, 0, 0], [2 ** 31 - 1, 2 ** 31 - 1, 3], table, queue, [7, 8, 0, 0], 16, 7)
    check_plan([64, 16, 17], [-1, 1, 1], np.arange(12).reshape(3, 4), np.arange(8), [6, 1, 0, 0], 16, 2)


def test_plan_after_a_refusal():
    """What comes after a sequence that was refused for its pages: without a new page it is served, with one it is not; and rows
    of long and short sequences that the batch's end cuts."""
    table, queue = np.arange(20).reshape(5, 4) % 12, np.arange(12)
    check_plan([14, 3, 30, 5, 16], [1, 40, 2, 3, 1], table, queue, [10, 2, 0, 0], 16, 60)
    check_plan([16, 3, 30, 5, 16], [1, 40, 2, 9, 1], table, queue, [10, 2, 0, 0], 16, 60)
    check_plan([16, 3, 30, 5, 16], [40, 1, 40, -1, 1], table, queue, [1, 0, 0, 0], 16, 90)
    for rows in range(1, 40):
        check_plan([5, 0, 16, 3, 7], [8, 9, 0, 12, 7], table, queue, [4, 12, 0, 0], 16, rows)
    rng = np.random.RandomState(9)
    for count in range(0, 9):
        seqs = 700
        lens, new = rng.randint(0, 40, seqs), rng.choice([0, 1, 1, 8, 9, -1], seqs, p=[.2, .3, .2, .1, .1, .1])
        check_plan(lens, new, rng.permutation(seqs * 4).reshape(seqs, 4), np.arange(3000), [2995, 40 * count, 0, 0], 16, 1200)


def test_plan_does_not_leave_its_buffers_whatever_they_hold():
    """Negative and huge lengths, ids outside the pool, a head and a count that are none: as if cut to the buffers."""
    rng = np.random.RandomState(1)
    for seed in range(4):
        lens = rng.choice([-5, 0, 3, 2 ** 31 - 1, 40], 50)
        new = rng.choice([-1, -2 ** 31, 1, 2, 2 ** 31 - 1], 50)
        guard = torch.full((3, 4096), 55, dtype=torch.int32, device="cuda")
        table, queue, slots = guard[0, 1000:1200].view(50, 4), guard[1, 1000:1017], guard[2, 1000:1060]
        table.copy_(dev(rng.choice([-7, 3, 10 ** 9], (50, 4))))
        queue.copy_(dev(rng.choice([-7, 3, 10 ** 9], 17)))
        out = [torch.empty(n, dtype=torch.int32, device="cuda") for n in (50, 51, 60, 60, 4)]
        out[2] = slots
        plan = binding.paged_plan(dev(lens), dev(new), table, queue, dev([[-3, 99, 0, 0], [16, -1, 0, 0], [2 ** 31 - 1, 17, 0, 0], [0, 9, 0, 0]][seed]), 16, out=out)
        torch.cuda.synchronize()
        for row, (a, b) in zip(guard, ((1000, 1200), (1000, 1017), (1000, 1060))):
            assert (row[:a] == 55).all() and (row[b:] == 55).all()
        assert ((plan.slots >= -1) & (plan.slots < 17 * 16)).all() and ((plan.lens >= 0) & (plan.lens <= 64)).all()
        assert 0 <= int(plan.state[0]) < 17 and 0 <= int(plan.state[1]) <= 17


# ---- write and read -------------------------------------------------------------------------------------------------

def make_pool(fmt, pages, G, D, page, seed=None):
    """A pool of random bytes (None: 0x55): what a page held before is nobody's business."""
    pool = binding.paged_pool(fmt, pages, G, D, page)
    for t in pool:
        t.copy_(torch.randint(0, 256, t.shape, dtype=torch.uint8, device="cuda", generator=torch.Generator("cuda").manual_seed(seed))
                if seed is not None else torch.full_like(t, 0x55))
    return pool


def host_pool(pool):
    return {n: t.cpu().numpy().copy() for n, t in zip(NAMES, pool)}


def activations(rng, rows, cols):
    x = rng.randn(rows, cols).astype(np.float32)
    x[:, rng.choice(cols, max(1, cols // 50), replace=False)] *= 40
    x[:, ::7] += 1
    return x


@pytest.mark.parametrize("name", FORMATS)
@pytest.mark.parametrize("H,G,D,page,rows", [(4, 2, 128, 16, 1), (12, 12, 64, 32, 37), (5, 1, 64, 64, 3), (32, 8, 128, 128, 130), (40, 8, 128, 1024, 6)])
def test_rows_written_as_the_oracle_and_the_separate_calls_have_them(name, H, G, D, page, rows):
    kind, asym = FORMATS[name]
    fmt = binding.make_format(kind, asym)
    rng = np.random.RandomState(rows)
    pages = max(3, 2 * rows // page)
    x = activations(rng, rows, (H + 2 * G) * D + 8)
    slots = rng.permutation(pages * page)[:rows].astype(np.int32)
    positions = rng.choice([0, 1, 77, 4095, 131071, 2 ** 30 - 1], rows).astype(np.int32)
    if rows > 2:
        slots[1] = -1                        # not stored
        slots[2] = pages * page              # one behind the last
        positions[1] = -1                    # its q is left as it was
    pool = make_pool(fmt, pages, G, D, page)
    want = host_pool(pool)
    q = torch.full((rows, H, D), 3.0, dtype=torch.bfloat16, device="cuda")
    got = binding.paged_write(fmt, torch.from_numpy(x).cuda(), pool, dev(slots), dev(positions), H, THETA, q=q)
    assert got is q
    want_q = paged_ref.write(x, want, slots, positions, H, THETA, kind, asym)
    want_q[positions < 0] = 0x4040
    np.testing.assert_array_equal(bits(q).reshape(rows, H, D), want_q)
    for n, t in zip(NAMES, pool):
        np.testing.assert_array_equal(t.cpu().numpy(), want[n], err_msg=n)   # the whole pool: nothing else was touched
    # the library's own separate calls: rotation, cast along the head dimension
    t = rows - 1 if rows != 3 else 0  # (a row that is stored)
    xs = torch.from_numpy(x[t:t + 1]).cuda()
    kc, ks = binding.split_heads_rope_quantize(fmt, xs, H * D, G, D, int(positions[t]), THETA)
    vc, vs = binding.quantize(fmt, binding.split_heads_rope(xs, (H + G) * D, G, D, False).view(G, D))
    p, o = int(slots[t]) // page, int(slots[t]) % page
    assert torch.equal(pool[0][p, :, o], kc[:, 0]) and torch.equal(pool[2][p, :, o], vc)
    assert torch.equal(pool[1][p, :, :, o], ks[:, 0]) and torch.equal(pool[3][p, :, :, o], vs.view_as(ks[:, 0]))
    assert torch.equal(q[t], binding.split_heads_rope(xs, 0, H, D, True, int(positions[t]), THETA)[:, 0])


@pytest.mark.parametrize("H,G,D,rows", [(3, 1, 64, 2051), (9, 2, 128, 2046), (1024, 1, 64, 3), (5, 1024, 64, 2)])
def test_rows_written_many_rows_and_many_heads(H, G, D, rows):
    """Long prompts, where a workgroup has all heads of its rows; and the most heads."""
    rng = np.random.RandomState(rows)
    kind, asym = FORMATS["amxfp4_e5m2"]
    fmt, pages, page = binding.make_format(kind, asym), -(-rows // 64) + 2, 64
    x = activations(rng, rows, (H + 2 * G) * D + 4)
    slots, positions = rng.permutation(pages * page)[:rows].astype(np.int32), rng.randint(0, 3 * 10 ** 5, rows).astype(np.int32)
    slots[rows // 2], positions[rows // 2] = -1, -1
    pool = make_pool(fmt, pages, G, D, page)
    want = host_pool(pool)
    q = torch.full((rows, H, D), 3.0, dtype=torch.bfloat16, device="cuda")
    binding.paged_write(fmt, torch.from_numpy(x).cuda(), pool, dev(slots), dev(positions), H, THETA, q=q)
    want_q = paged_ref.write(x, want, slots, positions, H, THETA, kind, asym)
    want_q[positions < 0] = 0x4040
    np.testing.assert_array_equal(bits(q).reshape(rows, H, D), want_q)
    for n, t in zip(NAMES, pool):
        np.testing.assert_array_equal(t.cpu().numpy(), want[n], err_msg=n)


@pytest.mark.parametrize("name", FORMATS)
@pytest.mark.parametrize("G,D,page,rows", [(2, 128, 16, 1), (12, 64, 32, 50), (1, 64, 256, 7), (8, 128, 64, 333)])
def test_rows_read_back(name, G, D, page, rows):
    kind, asym = FORMATS[name]
    fmt = binding.make_format(kind, asym)
    pages = 9
    pool = make_pool(fmt, pages, G, D, page, seed=3)
    for s in (pool[1], pool[3]):
        s.copy_(s % 0x78)  # finite scales
    slots = np.random.RandomState(rows).randint(-1, pages * page + 1, rows)
    slots[0] = pages * page - 1
    host = host_pool(pool)
    outs = binding.paged_read(fmt, pool, dev(slots)), binding.paged_read(fmt, pool, dev(slots), dtype=torch.float32)
    for i, n in enumerate("kv"):
        want = np.zeros((rows, G, D))
        for t, s in enumerate(slots):
            if 0 <= s < pages * page:
                want[t] = paged_ref.held(host, n, np.array([s // page] * 1024), s % page + 1, kind, asym)[0][-1]
        assert np.array_equal(f64(bits(outs[0][i])).reshape(want.shape), want)
        assert np.array_equal(outs[1][i].cpu().numpy().astype(np.float64), want)


def test_the_same_slot_twice_stays_inside_the_slot():
    fmt = binding.make_format()
    pool = make_pool(fmt, 4, 2, 64, 16)
    before = host_pool(pool)
    x = torch.randn(9, 6 * 64, device="cuda")
    binding.paged_write(fmt, x, pool, dev([21] * 9), dev(range(9)), 2, THETA)
    for n, t in zip(NAMES, pool):
        changed = np.argwhere(t.cpu().numpy() != before[n])
        place = 2 if n.endswith("codes") else 3
        assert len(changed) and (changed[:, 0] == 1).all() and (changed[:, place] == 5).all()


# ---- attention ------------------------------------------------------------------------------------------------------

def filled(rng, fmt_name, G, D, page, lens, width, pages=None, spoil=True):
    """A pool with the sequences' tokens in pages in no order, random bytes everywhere else (infinite and NaN scales among them)."""
    kind, asym = FORMATS[fmt_name]
    fmt = binding.make_format(kind, asym)
    count = [-(-n // page) for n in lens]
    pages = pages or sum(count) + 3
    ids = rng.permutation(pages)
    table, at = np.full((len(lens), width), -1 if not spoil else 10 ** 9), 0
    for b, c in enumerate(count):
        table[b, :c] = ids[at:at + c]
        at += c
    pool = make_pool(fmt, pages, G, D, page, seed=int(rng.randint(1000)))
    slots = np.concatenate([table[b, np.arange(n) // page] * page + np.arange(n) % page for b, n in enumerate(lens)] + [[]]).astype(np.int32)
    if len(slots):
        x = activations(rng, len(slots), (2 + 2 * G) * D)
        x[:, 2 * D:(2 + G) * D] *= 0.3 if D == 128 else 0.5
        positions = np.concatenate([np.arange(n) for n in lens])
        binding.paged_write(fmt, torch.from_numpy(x).cuda(), pool, dev(slots), dev(positions), 2, THETA)
    return fmt, pool, table


def allowed(want, weight, size, D):
    """How far an element may be off, from the roundings (weight: A below, size: B):
      - every weight times scale is rounded to BF16: half a step is 2^-8 of it, so the sum is off by at most 2^-8 of
        A = sum |weight V|;
      - a score is a sum of D <= 128 products in FP32, off by at most D 2^-24 B, B = scale sum |q k| at its largest, and by
        2^-22 of itself (<= B) for the two scalings; weights and their sum each take e^(that): A (2 B (D 2^-24 + 2^-22));
      - exp2, the running sums and factors, the merge: some 2^-21 of A each over at most 32 steps of rescaling: 2^-16 A;
      - the result is rounded to BF16 once: 2^-8 of its size (and of the error, hence 1 + 2^-8);
      - weights below 2^-126 become 0: with at most 2^13 tokens and values below 2^13 less than 2^-100."""
    return weight * (2.0 ** -8 + 2 * size * (D * 2.0 ** -24 + 2.0 ** -22) + 2.0 ** -16) * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(want) + 2.0 ** -100


def check_attention(rng, fmt_name, H, G, D, page, lens, rows, width=None, spare=0, positions=None, max_keys=0, table_of=None):
    """rows: how many of its newest tokens each sequence asks with."""
    kind, asym = FORMATS[fmt_name]
    width = width or max(1, -(-max(lens) // page))
    fmt, pool, table = filled(rng, fmt_name, G, D, page, lens, width)
    if table_of is not None:
        table = table_of(table)
    starts = np.concatenate([[0], np.cumsum(rows)])
    T = int(starts[-1]) + spare
    if positions is None:
        positions = np.concatenate([np.arange(n - r, n) for n, r in zip(lens, rows)] + [np.full(spare, -1)])
    q = torch.from_numpy(rng.randn(T, H, D).astype(np.float32)).to(torch.bfloat16).cuda()
    out = torch.full((T, H * D), 7.0, dtype=torch.bfloat16, device="cuda")
    need = binding.paged_attention_workspace_bytes(fmt, pool, T, H, len(lens), max_keys)
    ws = torch.full((need + 4096,), 0xFF, dtype=torch.uint8, device="cuda")  # (NaN wherever it is read before it is written)
    args = (fmt, q, pool, dev(table), dev(lens), dev(starts), dev(positions), 1 / math.sqrt(D))
    binding.paged_attention(*args, max_keys=max_keys, out=out, workspace=ws[:need])
    assert (ws[need:] == 0xFF).all()
    got = f64(bits(out)).reshape(T, H, D)
    want, weight, size = paged_ref.attention(f64(bits(q)).reshape(T, H, D), host_pool(pool), table, lens, starts, positions, 1 / math.sqrt(D), kind, asym)
    none = np.isnan(want)
    assert (got[none] == 7.0).all()                       # rows behind the last sequence's: as they were
    e = np.where(none, 0, got - want)
    worst = np.where(none, -1, np.abs(e) - allowed(want, weight, size[..., None], D))
    assert not np.isnan(e).any() and (worst <= 0).all(), (worst.max(), np.unravel_index(worst.argmax(), worst.shape))
    print("rel %.2e" % (np.linalg.norm(e) / max(1e-30, np.linalg.norm(np.where(none, 0, want)))))
    again = binding.paged_attention(*args, max_keys=max_keys, workspace=torch.zeros(need + 256, dtype=torch.uint8, device="cuda"))
    assert torch.equal(again[:starts[-1]], out[:starts[-1]])   # the same bits, whatever the workspace held
    return out


@pytest.mark.parametrize("name", FORMATS)
@pytest.mark.parametrize("H,G,D", [(8, 2, 128), (12, 12, 64), (16, 2, 128), (16, 2, 64)])
def test_attention_formats_and_heads(name, H, G, D):
    rng = np.random.RandomState(len(name) + D)
    check_attention(rng, name, H, G, D, 32, [1, 33, 200, 64, 129], [1] * 5)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256, 1024])
@pytest.mark.parametrize("D", [64, 128])
def test_attention_page_sizes_and_lengths(page, D):
    rng = np.random.RandomState(page + D)
    lens = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 700]
    check_attention(rng, "amxfp4_e5m2", 8, 2, D, page, lens, [0] + [1] * 17, width=70)


@pytest.mark.parametrize("H,G", [(1, 1), (3, 3), (4, 1), (5, 1), (7, 1), (8, 1), (9, 1), (16, 1), (17, 1), (24, 2), (64, 8)])
@pytest.mark.parametrize("D", [64, 128])
def test_attention_heads_to_a_key_head(H, G, D):
    rng = np.random.RandomState(H)
    check_attention(rng, "amxfp4_e5m2", H, G, D, 64, [100, 31, 5], [1, 1, 1])


@pytest.mark.parametrize("rows", [[1, 2, 3], [4, 4, 4], [8, 1, 0], [5, 0, 31], [0, 0, 70], [17, 33, 2]])
@pytest.mark.parametrize("H,G,D", [(8, 2, 128), (4, 4, 64), (40, 8, 128)])
def test_attention_several_rows_of_a_sequence(rows, H, G, D):
    rng = np.random.RandomState(sum(rows))
    check_attention(rng, "amxfp4_e5m2", H, G, D, 16, [max(r, 1) + n for r, n in zip(rows, (90, 3, 0))], rows, spare=2)


@pytest.mark.parametrize("lens,rows", [([5000], 1), ([2049, 1], 2), ([3000, 2999, 4097, 6], 1), ([9000], 4)])
@pytest.mark.parametrize("name,H,G,D", [("amxfp4_e5m2", 8, 2, 128), ("mxfp4_e8m0", 4, 4, 64)])
@pytest.mark.parametrize("known", [False, True])
def test_attention_long_and_split(lens, rows, name, H, G, D, known):
    rng = np.random.RandomState(len(lens) + rows)
    check_attention(rng, name, H, G, D, 64, lens, [min(rows, n) for n in lens], max_keys=max(lens) if known else 0)


@pytest.mark.parametrize("lens,rows,H,G", [([9000], 1, 16, 1), ([3100, 1, 2000], 1, 32, 2), ([6000], 5, 8, 2), ([2000] * 20, 1, 64, 4)])
def test_attention_long_with_all_columns_taken(lens, rows, H, G):
    """Sixteen combinations to a tile: parts of 2048 floats, joined by several workgroups where there are few segments."""
    check_attention(np.random.RandomState(H + rows), "amxfp4_e8m0", H, G, 128, 64, lens, [min(rows, n) for n in lens], spare=1)


@pytest.mark.parametrize("lens,rows,H,G,D,width", [
    ([2100, 5], [2000, 1], 4, 2, 64, 34), ([900, 0, 77], [900, 0, 77], 2, 1, 128, 15),   # chunks of prompts
    ([40, 3, 17], [1, 1, 1], 1024, 1, 64, 1), ([70, 3], [1, 2], 1024, 1024, 64, 2), ([1100], [1], 1024, 2, 128, 20),   # the most heads
    ([1 + b % 70 for b in range(4096)], [int(b % 2 == 0) for b in range(4096)], 1, 1, 64, 18)])   # the most sequences, split
def test_attention_at_the_limits(lens, rows, H, G, D, width):
    check_attention(np.random.RandomState(H + D), "amxfp4_e5m2", H, G, D, 64, lens, rows, width=width)


def test_attention_max_keys_too_small_costs_time_only():
    check_attention(np.random.RandomState(2), "amxfp4_e5m2", 8, 2, 128, 64, [3000, 40, 900], [1, 1, 2], max_keys=10)


def test_attention_many_sequences():
    rng = np.random.RandomState(3)
    lens = rng.randint(0, 150, 300)
    check_attention(rng, "mxfp4_e5m2", 4, 2, 64, 16, list(lens), [int(n > 0) for n in lens], spare=3)


def test_attention_most_sequences():
    lens = [1 + b % 5 for b in range(4096)]
    check_attention(np.random.RandomState(5), "amxfp4_e4m3", 2, 1, 64, 16, lens, [int(b % 3 == 0) for b in range(4096)])


@pytest.mark.parametrize("H,G,D,rows", [(16, 4, 128, 1), (32, 4, 128, 1), (64, 4, 128, 1), (12, 4, 128, 3), (16, 4, 64, 1), (64, 4, 64, 1)])
def test_attention_short_sequences_by_the_wave(H, G, D, rows):
    """More sequences and key heads than the card takes in workgroups, each for one wave: with every number of columns to a combination."""
    rng = np.random.RandomState(H + D)
    lens = list(rng.randint(1, 140, 258)) + [0, 280]
    check_attention(rng, "amxfp4_e5m2", H, G, D, 32, lens, [min(rows, n) for n in lens], spare=1)


@pytest.mark.parametrize("H,G,D,rows", [(8, 2, 128, 1), (4, 1, 64, 2), (16, 1, 128, 1)])
def test_attention_split_with_more_sequences_than_are_kept(H, G, D, rows):
    """Many sequences, most of them short, where the table has room for long ones."""
    rng = np.random.RandomState(H + rows)
    lens = list(rng.randint(0, 60, 700))
    lens[3], lens[650] = 1300, 2100
    check_attention(rng, "amxfp4_e5m2", H, G, D, 64, lens, [min(rows, n) for n in lens], width=34, spare=2)


def test_attention_rows_that_see_nothing_and_pages_outside_the_pool():
    rng = np.random.RandomState(4)
    lens, rows = [70, 200, 16, 300], [2, 1, 2, 1]
    positions = np.array([-1, 69, 199, -1, -1, 17])   # (the last sees 18 of its 300 tokens)

    def spoil(table):
        table = table.copy()
        table[1, :] = -1             # no page of the second sequence is in the pool
        table[3, 1] = 2 ** 31 - 1    # one of the last one's is not
        return table
    out = check_attention(rng, "amxfp4_e5m2", 4, 2, 128, 16, lens, rows, positions=positions, table_of=spoil)
    assert (out[[0, 2, 3, 4]] == 0).all() and (out[1] != 0).any()


@pytest.mark.parametrize("H,G,D", [(8, 2, 128), (32, 2, 128), (8, 8, 64)])
@pytest.mark.parametrize("width", [10, 80])
def test_attention_queries_of_rows_that_see_nothing_may_hold_anything(H, G, D, width):
    """Rows that were refused keep what their memory held: NaN and infinities there reach no other row and give zeros."""
    rng = np.random.RandomState(H)
    lens, rows = [70, 200, 0, 300], [3, 2, 1, 1]
    fmt, pool, table = filled(rng, "amxfp4_e5m2", G, D, 32, lens, width)
    starts, positions = np.concatenate([[0], np.cumsum(rows)]), np.array([-1, 68, -1, 198, -1, -1, 299])
    q = torch.from_numpy(rng.randn(7, H, D).astype(np.float32)).to(torch.bfloat16).cuda()
    spoiled = q.clone()
    spoiled[torch.from_numpy(positions < 0)] = torch.tensor([float("nan"), float("inf"), -float("inf"), 3e38] * (D // 4)).to(torch.bfloat16).cuda()
    a, b = (binding.paged_attention(fmt, x, pool, dev(table), dev(lens), dev(starts), dev(positions), 0.1) for x in (q, spoiled))
    assert torch.equal(a, b) and (a[torch.from_numpy(positions < 0)] == 0).all() and (a[torch.from_numpy(positions >= 0)] != 0).any(1).all()


def test_attention_beyond_four_gigabytes():
    """Codes at byte offsets over 2^32: the pages at the end of a large pool."""
    rng = np.random.RandomState(6)
    G, D, page = 8, 128, 256
    pages = (9 << 29) // (G * page * D // 2)   # 4.5 GiB of codes
    fmt = binding.make_format()
    pool = binding.paged_pool(fmt, pages, G, D, page)
    n = 600
    table = np.array([[pages - 1, 0, pages - 2]])
    slots = table[0][np.arange(n) // page] * page + np.arange(n) % page
    x = activations(rng, n, (8 + 2 * G) * D)
    x[:, 8 * D:16 * D] *= 0.3
    q = binding.paged_write(fmt, torch.from_numpy(x).cuda(), pool, dev(slots), dev(np.arange(n)), 8, THETA)
    out = binding.paged_attention(fmt, q[-1:].contiguous(), pool, dev(table), dev([n]), dev([0, 1]), dev([n - 1]), 0.088)
    k, v = (t.double() for t in binding.paged_read(fmt, pool, dev(slots)))
    s = torch.einsum("hd,jhd->hj", q[-1].double(), k) * float(np.float32(0.088))
    w = torch.softmax(s, -1)
    want, weight = (torch.einsum("hj,jhd->hd", w, y).reshape(1, -1) for y in (v, v.abs()))
    # (the two roundings to BF16, half a step each, and a 64th of that for everything in FP32)
    assert ((out.double() - want).abs() <= 2.0 ** -8 * (1 + 2.0 ** -6) * (weight + want.abs())).all()
    c, sc = ref.quantize(paged_ref.bf16_from_f32(x[-1:, 16 * D:].reshape(G, D)), 32, ref.FP8_E5M2, True)
    assert np.array_equal(v[-1].cpu().numpy(), ref.dequantize(c, sc))


# ---- together -------------------------------------------------------------------------------------------------------

class Server:
    """What a serving program keeps for a batch of conversations, and one step of it."""

    def __init__(self, fmt, H, G, D, seqs, width, pages, page, rows):
        i = dict(dtype=torch.int32, device="cuda")
        self.fmt, self.H, self.page = fmt, H, page
        self.pool = make_pool(fmt, pages, G, D, page, seed=1)
        self.table, self.queue = torch.full((seqs, width), -1, **i), torch.randperm(pages, device="cuda").int()
        self.lens, self.state = torch.zeros(seqs, **i), torch.tensor([0, pages, 0, 0], **i)
        self.new = torch.zeros(seqs, **i)
        self.plan = binding.PagedPlan(*(torch.zeros(n, **i) for n in (seqs, seqs + 1, rows, rows, 4)))
        self.proj = torch.zeros((rows, (H + 2 * G) * D), device="cuda")
        self.q = torch.zeros((rows, H, D), dtype=torch.bfloat16, device="cuda")
        self.out = torch.zeros((rows, H * D), dtype=torch.bfloat16, device="cuda")
        self.ws = torch.empty(binding.paged_attention_workspace_bytes(fmt, self.pool, rows, H, seqs, 0), dtype=torch.uint8, device="cuda")
        self.scale = 1 / math.sqrt(D)

    def step(self):
        p = binding.paged_plan(self.lens, self.new, self.table, self.queue, self.state, self.page, out=self.plan)
        binding.paged_write(self.fmt, self.proj, self.pool, p.slots, p.positions, self.H, THETA, q=self.q)
        binding.paged_attention(self.fmt, self.q, self.pool, self.table, p.lens, p.starts, p.positions, self.scale, out=self.out, workspace=self.ws)
        self.lens.copy_(p.lens)
        self.state.copy_(p.state)


def dense(history, rows, H, G, D, scale, kind, asym):
    """The newest `rows` rows of one conversation, all of whose projections are `history`, in float64; and what it may be
    off by: check_attention()'s bound (the outlier columns make scores of several hundred, so their own FP32 error counts)."""
    n = len(history)
    x = history.reshape(n, H + 2 * G, D)
    turned = paged_ref.rotate(x[:, :H + G], np.arange(n), THETA)
    kv = []
    for y in (turned[:, H:], paged_ref.bf16_from_f32(x[:, H + G:])):
        c, s = ref.quantize(np.ascontiguousarray(y.reshape(-1, D)), 32, kind, asym)
        kv.append(ref.dequantize(c, s, 32, kind, asym).reshape(n, G, D))
    out, tol = np.zeros((rows, H, D)), np.zeros((rows, H, D))
    for i in range(rows):
        m = n - rows + i + 1
        for h in range(H):
            s = kv[0][:m, h // (H // G)] @ f64(turned[m - 1, h]) * scale
            w = np.exp(s - s.max())
            out[i, h] = (w / w.sum()) @ kv[1][:m, h // (H // G)]
            size = scale * np.max(np.abs(kv[0][:m, h // (H // G)]) @ np.abs(f64(turned[m - 1, h])))
            weight = (w / w.sum()) @ np.abs(kv[1][:m, h // (H // G)])
            tol[i, h] = allowed(out[i, h], weight, size, D)
    return out.reshape(rows, -1), tol.reshape(rows, -1)


@pytest.mark.parametrize("captured", [False, True])
def test_conversations_step_by_step(captured):
    """Prompts of different lengths, single tokens, drafts, an idle conversation, one that ends and whose pages others take, one
    that is refused: every row against the textbook attention over its whole history. Captured: each step is a replay of one
    graph (other lengths, same buffers), with eager work between the replays."""
    H, G, D, seqs, page, rows = 8, 2, 64, 5, 16, 48
    kind, asym = FORMATS["amxfp4_e5m2"]
    fmt = binding.make_format(kind, asym)
    s = Server(fmt, H, G, D, seqs, 8, 11, page, rows)
    history = [np.zeros((0, (H + 2 * G) * D), np.float32) for _ in range(seqs)]
    rng = np.random.RandomState(0)
    graph = None
    if captured:
        s.step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            s.step()
    refused = 0
    for new in ([20, 1, 0, 17, 3], [1, 1, 1, 1, 1], [4, 0, 3, 1, -1], [1, 30, 1, 1, 9], [1, 1, 1, -1, 30], [1, 1, 1, 0, 12], [1, 1, 40, 5, 1],
                [1, -1, 40, 5, 1], [1, 2, 1, 0, 1]):
        x = activations(rng, rows, (H + 2 * G) * D)
        s.new.copy_(dev(new))
        s.proj.copy_(torch.from_numpy(x).cuda())
        s.out.fill_(7.0)
        before = s.lens.cpu().numpy()
        graph.replay() if captured else s.step()
        torch.cuda.synchronize()
        got, lens, starts = f64(bits(s.out)).reshape(rows, -1), s.plan.lens.cpu().numpy(), s.plan.starts.cpu().numpy()
        for b, n in enumerate(new):
            mine = got[starts[b]:starts[b + 1]]
            if n < 0:
                history[b] = history[b][:0]
            elif n > 0 and lens[b] == before[b]:
                refused += 1
                assert (mine == 0).all()
            elif n > 0:
                history[b] = np.concatenate([history[b], x[starts[b]:starts[b + 1]]])
                want, tol = dense(history[b], n, H, G, D, s.scale, kind, asym)
                worst = np.abs(mine - want) - tol
                at = np.unravel_index(worst.argmax(), worst.shape)
                assert (worst <= 0).all(), (new, b, len(history[b]), [float(v) for v in (*at, mine[at], want[at], tol[at])], int((worst > 0).sum()))
            assert lens[b] == len(history[b])
        assert (got[starts[-1]:] == 7.0).all()
        torch.randn(1000, device="cuda").sum().item()   # eager work between the replays
    assert refused >= 1


def test_on_another_stream():
    fmt = binding.make_format()
    a, b = (Server(fmt, 4, 2, 64, 3, 4, 20, 16, 30) for _ in range(2))
    b.queue.copy_(a.queue)
    b.pool = binding.PagedPool(*(t.clone() for t in a.pool))
    side = torch.cuda.Stream()
    for step in range(3):
        x = torch.randn_like(a.proj)
        for s in (a, b):
            s.new.copy_(dev([9, 1, 5]))
            s.proj.copy_(x)
        a.step()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            b.step()
        side.synchronize()
        assert torch.equal(a.out, b.out) and torch.equal(a.lens, b.lens)


def test_the_native_way_and_the_general_one(monkeypatch):
    """With all buffers given the calls go through the native module, and give what the general way gives."""
    fmt = binding.make_format()
    a, b = (Server(fmt, 4, 2, 128, 3, 4, 20, 16, 30) for _ in range(2))
    b.queue.copy_(a.queue)
    b.pool = binding.PagedPool(*(t.clone() for t in a.pool))
    taken = []

    class Spy:
        def __getattr__(self, name):
            def call(*args):
                rc = getattr(calls, name)(*args)
                taken.append((name, rc))
                return rc
            return call
    binding.load()
    calls = binding._calls
    for s, module in ((a, Spy()), (b, binding._GeneralWay())):
        monkeypatch.setattr(binding, "_calls", module)
        s.proj.copy_(torch.arange(s.proj.numel(), device="cuda").view_as(s.proj) % 37 - 15.5)
        s.new.copy_(dev([9, 1, 5]))
        s.step()
        k = torch.zeros(30, 2, 128, dtype=torch.bfloat16, device="cuda")
        s.kv = binding.paged_read(fmt, s.pool, s.plan.slots, k=k, v=k.clone())
    assert taken == [("paged_plan", 0), ("paged_write", 0), ("paged_attention", 0), ("paged_read", 0)]
    for x, y in zip((a.out, a.q, a.table, a.queue, *a.plan, *a.pool, *a.kv), (b.out, b.q, b.table, b.queue, *b.plan, *b.pool, *b.kv)):
        assert torch.equal(x, y)


def test_binding_refuses_what_does_not_fit():
    fmt = binding.make_format()
    s = Server(fmt, 4, 2, 64, 3, 4, 20, 16, 30)
    p = s.plan
    at = lambda **kw: binding.paged_attention(*[{**dict(fmt=fmt, q=s.q, pool=s.pool, table=s.table, lens=p.lens, starts=p.starts,  # noqa: E731
                                                      positions=p.positions, scale=0.1), **kw}[k] for k in
                                                 ("fmt", "q", "pool", "table", "lens", "starts", "positions", "scale")],
                                               out=kw.get("out"), workspace=kw.get("workspace"))
    for kw in (dict(q=s.q.float()), dict(q=s.q[:, :, :32]), dict(q=s.q[:, :3].contiguous()), dict(table=s.table.long()), dict(table=s.table[:2]),
               dict(lens=p.lens[:2]), dict(starts=p.starts[:3]), dict(positions=p.positions[:29]), dict(positions=p.positions.long()),
               dict(out=s.out.float()), dict(out=s.out[:29]), dict(pool=s.pool[:2] + s.pool[:2][::-1]),
               dict(pool=(s.pool[0], s.pool[1][..., 0].contiguous(), s.pool[2], s.pool[3][..., 0].contiguous())),
               dict(q=s.q.transpose(0, 1)), dict(fmt=binding.make_format(asymmetric=False)), dict(fmt=binding.make_format(group_size=16))):
        with pytest.raises(binding.AmxError):
            at(**kw)
    if s.ws.numel():
        with pytest.raises(binding.AmxError):
            at(workspace=s.ws[:-256])
    for call in (lambda: binding.paged_plan(p.lens, s.new, s.table, s.queue, s.state, 16, out=p),   # lens_out is lens
                 lambda: binding.paged_plan(s.lens, s.new, s.table, s.queue, s.state, 16),           # neither rows nor out
                 lambda: binding.paged_plan(s.lens, s.new[:2], s.table, s.queue, s.state, 16, out=p),
                 lambda: binding.paged_plan(s.lens, s.new, s.table, s.queue, s.state[:3], 16, out=p),
                 lambda: binding.paged_plan(s.lens, s.new, s.table.t(), s.queue, s.state, 16, out=p),
                 lambda: binding.paged_plan(s.lens, s.new, s.table, s.queue, s.state, 24, out=p),
                 lambda: binding.paged_write(fmt, s.proj.half(), s.pool, p.slots, p.positions, 4, THETA),
                 lambda: binding.paged_write(fmt, s.proj, s.pool, p.slots[:9], p.positions, 4, THETA),
                 lambda: binding.paged_write(fmt, s.proj, s.pool, p.slots, p.positions, 6, THETA),
                 lambda: binding.paged_write(fmt, s.proj, s.pool, p.slots, p.positions, 4, THETA, q=s.q[:3]),
                 lambda: binding.paged_write(fmt, s.proj.t(), s.pool, p.slots, p.positions, 4, THETA),
                 lambda: binding.paged_read(fmt, s.pool, p.slots.long()),
                 lambda: binding.paged_read(fmt, s.pool, p.slots, dtype=torch.float16),
                 lambda: binding.paged_read(fmt, s.pool, p.slots, k=s.out)):
        with pytest.raises(binding.AmxError):
            call()
