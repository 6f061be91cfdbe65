"""Oracle of the scoring operators (include/amxfp4_scoring.h): plain NumPy float64 (TEST INFRASTRUCTURE: only tests/ may import this;
it shares no code with the HIP path). Each function also says how far the float32 evaluation of the same formulas may be off."""
import numpy as np

from . import ref

TILE = 32


def score(s, cap, slope, distance):
    """s, capped, less slope for each key of distance."""
    if cap:
        s = cap * np.tanh(s / cap)
    return s - slope * distance


def ranges(Sq, Sk, causal, pos0, first, last):
    """(lo, hi) [Sq]: the first and the last key that each row sees; hi < lo where it sees none."""
    at = pos0 + np.arange(Sq, dtype=np.int64)
    lo = np.zeros(Sq, np.int64) if first is None else np.maximum(np.asarray(first, np.int64), 0)
    hi = np.full(Sq, Sk - 1) if last is None else np.minimum(np.asarray(last, np.int64), Sk - 1)
    return lo, np.minimum(hi, at) if causal else hi


def cast_weights(p, scale_format, asymmetric):
    """Rows of 32 weights, each cast as one group and dequantized."""
    c, s = ref.quantize_f32(np.ascontiguousarray(p, np.float32), TILE, scale_format, asymmetric)
    return ref.dequantize(c, s, TILE, scale_format, asymmetric)


def cast_between(p, delta, scale_format, asymmetric, near=0.0):
    """How far apart the casts of weights within the relative error delta of p [32] may lie, element by element: the scale is that of the
    group's largest (1 +- delta; exactly 1 where it holds the running maximum), an element is monotone in the weight where the scale is given.
    near: a largest weight that is so near below 1 counts as 1 (what ties in exact arithmetic need not in FP32)."""
    values = []
    for top in (1.0,) if p.max() == 1 else (1 - delta, 1 + delta) + ((1 / p.max(),) if p.max() >= 1 - near else ()):
        for own in (1 - delta, 1.0, 1 + delta):
            q = p * own
            q[np.argmax(p)] = p.max() * top
            # (an element may not raise the scale: only the largest does)
            values.append(cast_weights(np.minimum(q, p.max() * top)[None], scale_format, asymmetric)[0])
    return np.max(values, 0) - np.min(values, 0)


def masked_attention(q_bits, k_bits, v_bits, scale, causal=True, pos0=0, first=None, last=None, cap=0.0, slopes=None,
                     scale_format=ref.FP8_E5M2, asymmetric=True, rows=None):
    """BF16 bit patterns q [Hq, Sq, D], k and v [Hkv, Sk, D]. Returns (out, allowed) float64 [Sq, Hq, D]; rows: only these (NaN elsewhere).

    allowed, for a BF16 result out of FP32 arithmetic:
      - a score is a sum of D products, off by D 2^-24 B (B = scale sum |q k|); scaling, tanh (2^-22 of the cap) and distances add 2^-22 of
        (B + cap + slope distance) each; exp2 and its argument 2^-22: a weight is off by delta, relatively, twice that for a difference of scores;
      - a weight next to a rounding boundary of the cast may fall on either side: cast_between(); a tile's largest score within 2^-16 + 2^-22
        of its size (in log2) of the running maximum counts as it;
      - the sums: 2^-22 for each tile's steps, a factor's argument 2^-23 of the largest score (in log2) each time the maximum moves;
      - the BF16 result: half a step, 2^-8 of it."""
    Hq, Sq, D = q_bits.shape
    Hkv, Sk, _ = k_bits.shape
    per = Hq // Hkv
    out, allowed = np.full((Sq, Hq, D), np.nan), np.full((Sq, Hq, D), np.nan)
    lo, hi = ranges(Sq, Sk, causal, pos0, first, last)
    kv = []
    for g in range(Hkv):
        kc, ks = ref.quantize(np.ascontiguousarray(k_bits[g]), 32, scale_format, asymmetric)
        vc, vs = ref.quantize(np.ascontiguousarray(v_bits[g]), 32, scale_format, asymmetric, k_axis=0)
        kv.append((ref.dequantize(kc, ks, 32, scale_format, asymmetric), ref.dequantize(vc, vs, 32, scale_format, asymmetric).T))
    sc = np.float64(np.float32(scale))
    for h in range(Hq):
        qc, qs = ref.quantize(np.ascontiguousarray(q_bits[h]), 32, scale_format, asymmetric)
        qh = ref.dequantize(qc, qs, 32, scale_format, asymmetric)
        kh, vh = kv[h // per]
        slope = 0.0 if slopes is None else np.float64(np.float32(slopes[h]))
        for i in range(Sq) if rows is None else rows:
            out[i, h], allowed[i, h] = 0.0, 0.0
            if hi[i] < lo[i]:
                continue
            j = np.arange(lo[i], hi[i] + 1)
            away = np.abs(pos0 + i - j).astype(np.float64)
            s = np.full(Sk, -np.inf)
            s[j] = score((kh[j] @ qh[i]) * sc, np.float64(np.float32(cap)), slope, away)
            B = float(np.max(np.abs(kh[j]) @ np.abs(qh[i])) * sc)
            # (distances count from the nearest key that is seen: a shift of the whole row)
            far = abs(slope) * float((away - away.min()).max())
            delta = 2 * (D * 2.0 ** -24 * B + 2.0 ** -22 * (B + cap + far)) + 2.0 ** -21
            m, l, o, slack, weight, tiles = -np.inf, 0.0, np.zeros(D), np.zeros(D), np.zeros(D), 0
            for t0 in range(lo[i] // TILE * TILE, hi[i] + 1, TILE):
                tile = s[t0:t0 + TILE]
                m_new = max(m, float(tile.max()))
                alpha, p = np.exp(m - m_new), np.exp(tile - m_new).astype(np.float32).astype(np.float64)
                p_hat = cast_weights(p[None], scale_format, asymmetric)[0]
                v = vh[t0:t0 + TILE]
                l, o = l * alpha + p.sum(), o * alpha + p_hat @ v
                near = 2.0 ** -16 + 2.0 ** -22 * 1.5 * (B + cap + far) + delta
                slack = slack * alpha + cast_between(p, delta, scale_format, asymmetric, near) @ np.abs(v)
                weight = weight * alpha + p_hat @ np.abs(v)
                m, tiles = m_new, tiles + 1
            out[i, h] = o / l
            e = slack / l + weight / l * (delta + (tiles + 8) * 2.0 ** -22 + tiles * 2.0 ** -23 * 1.5 * (B + cap + far))
            allowed[i, h] = e * (1 + 2.0 ** -7) + 2.0 ** -8 * np.abs(out[i, h]) + 2.0 ** -100
    return out, allowed


def paged_attention(q, pool, table, lens, starts, positions, softmax_scale, scale, asym, cap, slopes):
    """paged_ref.attention() with the scores above: (out, weight, size), size also of the cap and of the distances' share of a score."""
    from . import paged_ref
    rows, H, D = q.shape
    G = pool["k_codes"].shape[1]
    page, width = pool["k_codes"].shape[2], table.shape[1]
    out, weight, size = np.full((rows, H, D), np.nan), np.full((rows, H, D), np.nan), np.zeros((rows, H))
    for b in range(len(lens)):
        n = int(max(0, min(lens[b], width * page)))
        k, good = paged_ref.held(pool, "k", table[b], n, scale, asym)
        v, _ = paged_ref.held(pool, "v", table[b], n, scale, asym)
        for t in range(max(0, starts[b]), min(starts[b + 1], rows)):
            m = min(n, int(positions[t]) + 1)
            seen = np.flatnonzero(good[:max(m, 0)])
            for h in range(H):
                out[t, h] = weight[t, h] = 0
                if len(seen) == 0:
                    continue
                g = h // (H // G)
                slope = 0.0 if slopes is None else np.float64(np.float32(slopes[h]))
                away = (m - 1 - seen).astype(np.float64)
                s = score(k[seen, g] @ q[t, h] * np.float64(np.float32(softmax_scale)), np.float64(np.float32(cap)), slope, away)
                w = np.exp(s - s.max())
                w /= w.sum()
                out[t, h] = w @ v[seen, g]
                weight[t, h] = w @ np.abs(v[seen, g])
                size[t, h] = np.max(np.abs(k[seen, g]) @ np.abs(q[t, h])) * softmax_scale + cap + abs(slope) * away.max()
    return out, weight, size


def allowed_logprobs(p, z, vocab, cap):
    """(of a log probability, of an entropy), as token_logprobs() counts them; z: distances from the largest value, p: their probabilities."""
    segments = -(-min(-(-(vocab + 7) // 1024), 512) // 4)  # of a wave
    s = 16 * segments * 2.0 ** -24 + segments * 7 * 2.0 ** -24 + 30 * 5 * 2.0 ** -24 + 2.0 ** -21
    with np.errstate(over="ignore", invalid="ignore"):
        counts = p > 0
        A, Q = (p[counts] * -z[counts]).sum(), (p[counts] * z[counts] ** 2).sum()
    value = 1.25 * 2.0 ** -21 * cap
    of_s = s + value + A * 2.0 ** -22  # relative, of the sum
    # of the sum of exponentials times distances, over the sum
    of_t = value + A * (s + value + 2.0 ** -22) + Q * 2.0 ** -22
    return of_s + value, of_s + of_t + A * of_s


def token_logprobs(logits, targets, top, cap):
    """float64 logits [rows, vocab]. Returns (logprob, entropy, top_logprobs, top_ids, allowed of a log probability, allowed of an entropy).

    allowed, in the order of a thread's work, with z = x - m the distance from the largest value, A = sum p |z| and Q = sum p z^2:
      - a value is off by 2^-22 of the cap (a quarter more where tanh is near -1), a distance by two of those and 2^-24 of itself, an exponential by that,
        the rounding of its argument and 2^-22; a thread's maximum moves on from 0 to m in steps, whose factors' arguments add up to |z| again;
      - a thread reads every fourth of at most 512 segments of 1024 values, 16 of each, one after another: a rounding of 2^-24 to each, for the sum of
        exponentials and that of exponentials times distances, which both have terms of one sign; and with each segment a factor (2^-22) and up to
        three roundings;
      - some 30 joins (64 lanes, 4 waves, 64 parts) of 2^-22 and 2^-24 each; the logarithm and what is added behind it 2^-21."""
    rows, vocab = logits.shape
    live = logits > -np.inf
    with np.errstate(invalid="ignore", over="ignore"):
        x = cap * np.tanh(logits / cap) if cap else logits.copy()
    x[~live] = -np.inf
    logprob, entropy = np.zeros(rows), np.zeros(rows)
    tops, ids = np.zeros((rows, top)), np.zeros((rows, top), np.int64)
    off, off_entropy = np.zeros(rows), np.zeros(rows)
    for r in range(rows):
        y, seen = x[r], live[r]
        ids[r] = np.argsort(-logits[r], kind="stable")[:top]
        inside = targets is not None and 0 <= targets[r] < vocab
        if not seen.any():
            tops[r] = -np.inf
            logprob[r] = -np.inf if inside else 0.0
            continue
        m = y[seen].max()
        z = y - m
        lse = np.log(np.exp(z[seen]).sum())
        distance, z = z, z - lse
        logprob[r] = z[targets[r]] if inside else 0.0
        p = np.exp(z[seen])
        entropy[r] = -(p * z[seen]).sum()
        tops[r] = z[ids[r]]
        off[r], off_entropy[r] = allowed_logprobs(p, distance[seen], vocab, cap)
    return logprob, entropy, tops, ids, off, off_entropy
