"""Oracle of the paged key / value cache (TEST INFRASTRUCTURE, as the rest of this package): the bookkeeping of a step in plain
integers, sequence by sequence; the rows written, through the quantization oracle; the attention in float64. Pools are
dicts of uint8 arrays in the library's layout:
  codes [pages, kv_heads, page_size, head_dim / 2], scales [pages, kv_heads, head_dim / 32, page_size(, 2)]."""
import numpy as np

from . import ref


def plan(lens, new_rows, table, queue, state, page, rows):
    """Returns (lens, starts, slots, positions, state, table, queue) after the step; the arguments are left alone."""
    table, queue = np.array(table, np.int64), np.array(queue, np.int64)
    pages, width = len(queue), table.shape[1]
    head, count = int(state[0]) % pages, max(0, min(int(state[1]), pages))
    tail = head + count
    out_lens, starts, slots, positions, refused = [], [0], [-1] * rows, [-1] * rows, 0
    wanted, taken, given, begin = 0, 0, 0, 0
    for b, n in enumerate(int(v) for v in new_rows):
        have = max(0, min(int(lens[b]), width * page))
        held = -(-have // page)
        more = max(n, 0)
        fits = n > 0 and have + n <= width * page and begin + n <= rows
        if fits:
            want = -(-(have + n) // page) - held
            wanted += want
            if want and wanted <= count:
                for j in range(want):
                    table[b, held + j] = queue[(head + wanted - want + j) % pages]
                taken = wanted
            fits = want == 0 or wanted <= count
        if fits:
            for i in range(n):
                at = have + i
                positions[begin + i] = at
                p = table[b, at // page]
                slots[begin + i] = int(p) * page + at % page if 0 <= p < pages else -1
        refused += n > 0 and not fits
        out_lens.append(0 if n < 0 else have + n if fits else have)
        begin += more
        starts.append(min(begin, rows))
    given_ids = [table[b, j] for b, n in enumerate(new_rows) if n < 0 for j in range(-(-max(0, min(int(lens[b]), width * page)) // page))]
    for given, p in enumerate(given_ids):
        queue[(tail + given) % pages] = p
    state = [(head + taken) % pages, count - taken + len(given_ids), refused, starts[-1]]
    return tuple(np.array(v, np.int32) for v in (out_lens, starts, slots, positions, state, table, queue))


def bf16_from_f32(x):
    u = np.ascontiguousarray(x, np.float32).view(np.uint32)
    return ((u + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint16)


def rotate(x, positions, theta):
    """x [rows, heads, D] float32 -> BF16 bits of the rotated heads; angles, sines and products in float64, rounded to float32
    and then to BF16."""
    half = x.shape[-1] // 2
    ang = np.asarray(positions, np.float64)[:, None] * np.exp(-np.log(np.float64(theta)) * np.arange(half) / half)
    cs, sn = np.cos(ang)[:, None], np.sin(ang)[:, None]
    a, b = x[..., :half].astype(np.float64), x[..., half:].astype(np.float64)
    return bf16_from_f32(np.concatenate([a * cs - b * sn, b * cs + a * sn], -1).astype(np.float32))


def write(proj, pool, slots, positions, q_heads, theta, scale, asym):
    """Stores the rows in `pool` (in place) and returns the BF16 bits of the queries [rows, q_heads, D]."""
    pages, G, page, half = pool["k_codes"].shape
    D = 2 * half
    x = np.asarray(proj, np.float32)[:, :(q_heads + 2 * G) * D].reshape(len(slots), q_heads + 2 * G, D)
    turned = rotate(x[:, :q_heads + G], positions, theta)
    for name, y in (("k", turned[:, q_heads:]), ("v", bf16_from_f32(x[:, q_heads + G:]))):
        codes, scales = ref.quantize(np.ascontiguousarray(y.reshape(-1, D)), 32, scale, asym)
        codes = codes.reshape(len(slots), G, half)
        scales = scales.reshape((len(slots), G, D // 32) + ((2,) if asym else ()))
        for t, s in enumerate(slots):
            if 0 <= s < pages * page:
                pool[name + "_codes"][s // page, :, s % page] = codes[t]
                pool[name + "_scales"][s // page, :, :, s % page] = scales[t]
    return turned[:, :q_heads]


def held(pool, name, table_row, count, scale, asym):
    """What the first `count` tokens of a sequence are in the cache: float64 [count, kv_heads, D], and which of them lie in pages of
    the pool (the others are zeros)."""
    codes, scales = pool[name + "_codes"], pool[name + "_scales"]
    pages, G, page, half = codes.shape
    if count == 0:
        return np.zeros((0, G, 2 * half)), np.zeros(0, bool)
    j = np.arange(count)
    ids = np.asarray(table_row, np.int64)[j // page]
    good = (ids >= 0) & (ids < pages)
    ids = np.where(good, ids, 0)
    c = codes[ids, :, j % page].reshape(-1, half)
    s = scales[ids, :, :, j % page]
    x = ref.dequantize(c, s.reshape((c.shape[0],) + s.shape[2:]), 32, scale, asym).reshape(count, G, 2 * half)
    return np.where(good[:, None, None], x, 0.0), good


def attention(q, pool, table, lens, starts, positions, softmax_scale, scale, asym):
    """q [rows, heads, D] float64. Returns float64 (out, weight, size) [rows, heads, D], [rows, heads, D], [rows, heads]: the result;
    the sums of |weight * value| that errors of the weights are relative to; the largest scaled sum of |q k| that an error of a
    score is relative to. Rows of no sequence are NaN."""
    rows, H, D = q.shape
    G = pool["k_codes"].shape[1]
    page, width = pool["k_codes"].shape[2], table.shape[1]
    out, weight, size = np.full((rows, H, D), np.nan), np.full((rows, H, D), np.nan), np.zeros((rows, H))
    for b in range(len(lens)):
        n = int(max(0, min(lens[b], width * page)))
        k, good = held(pool, "k", table[b], n, scale, asym)
        v, _ = held(pool, "v", table[b], n, scale, asym)
        for t in range(max(0, starts[b]), min(starts[b + 1], rows)):
            m = min(n, int(positions[t]) + 1)
            seen = np.flatnonzero(good[:max(m, 0)])
            for h in range(H):
                out[t, h] = weight[t, h] = 0
                if len(seen) == 0:
                    continue
                g = h // (H // G)
                s = k[seen, g] @ q[t, h] * np.float64(np.float32(softmax_scale))
                w = np.exp(s - s.max())
                w /= w.sum()
                out[t, h] = w @ v[seen, g]
                weight[t, h] = w @ np.abs(v[seen, g])
                size[t, h] = np.max(np.abs(k[seen, g]) @ np.abs(q[t, h])) * softmax_scale
    return out, weight, size
