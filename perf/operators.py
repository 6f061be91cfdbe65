"""The paged key / value cache and the attention that reads it, as cases that can be timed and compared: what a serving
program calls for every step of a batch of conversations of different lengths.

    plan         pages from a queue, block tables, slots and positions of the new rows, from the lengths of the sequences
    write        rotary embedding of the new queries and keys, cast of keys and values into their slots; read back as values
    attention    queries of the new rows against everything that their sequences have in the cache
    step         the three one after the other, as a decoder layer makes them

    listed()              the named cases
    draw(rng)             one more case of the same ranges (rng: random.Random)
    prepare(case, seed)   the inputs, the cache and the buffers a serving program keeps, on the GPU
    run(state)            one pass: plain torch where `own` is false, the library's calls where it is true
    work(case)            bytes and floating-point operations the pass cannot do without
    exact(case, seed)     the outputs in 64 bits, sequence by sequence
"""
import functools
import math
import random

import torch

own = False
DEV = "cuda"
THETA = 500000.0
SCRATCH = 64 << 20  # bytes of scratch memory that a program keeps for the attention

# name -> (scale format, sign-asymmetric); groups of 32 along the head dimension
FORMATS = {
    "amxfp4_e5m2": ("e5m2", True),
    "mxfp4_e5m2": ("e5m2", False),
    "amxfp4_e4m3": ("e4m3", True),
    "amxfp4_e8m0": ("e8m0", True),
    "mxfp4_e8m0": ("e8m0", False),
}


def listed():
    return [
        # every conversation of a small batch gets one token, a few have just ended: launches are all there is
        {"name": "plan_64", "kind": "plan", "seqs": 64, "keys": 16384, "page": 64, "rows": 1, "spare": 3, "short": False},
        # a large server: a thousand slots, chunks of prompts among single tokens, small pages, and not enough of them
        {"name": "plan_1000_mixed", "kind": "plan", "seqs": 1000, "keys": 8000, "page": 16, "rows": 48, "spare": 100, "short": True},
        # the new token of one conversation
        {"name": "write_1", "kind": "write", "fmt": "amxfp4_e5m2", "heads": 32, "kv_heads": 8, "head_dim": 128, "seqs": 1,
         "keys": 8192, "page": 64, "rows": 1, "spare": 0},
        # one token each of a batch of 256, 70B-shaped heads
        {"name": "write_256", "kind": "write", "fmt": "amxfp4_e5m2", "heads": 64, "kv_heads": 8, "head_dim": 128, "seqs": 256,
         "keys": 1500, "page": 32, "rows": 1, "spare": 0},
        # prompts of 23 conversations packed into one prefill, power-of-two scales
        {"name": "write_23_prompts", "kind": "write", "fmt": "amxfp4_e8m0", "heads": 32, "kv_heads": 8, "head_dim": 128, "seqs": 23,
         "keys": 900, "page": 128, "rows": 600, "spare": 17},
        # one conversation of some paragraphs, the next token
        {"name": "attention_1x700", "kind": "attention", "fmt": "amxfp4_e5m2", "heads": 32, "kv_heads": 8, "head_dim": 128, "seqs": 1,
         "keys": 700, "page": 64, "rows": 1, "spare": 0},
        # 64 conversations of up to 16384 tokens, the next token of each: bound by reading the cache
        {"name": "attention_64x16384", "kind": "attention", "fmt": "amxfp4_e5m2", "heads": 32, "kv_heads": 8, "head_dim": 128,
         "seqs": 64, "keys": 16384, "page": 64, "rows": 1, "spare": 0},
        # one long document, the next token of its answer
        {"name": "attention_1x131000", "kind": "attention", "fmt": "amxfp4_e5m2", "heads": 32, "kv_heads": 8, "head_dim": 128, "seqs": 1,
         "keys": 131000, "page": 256, "rows": 1, "spare": 0},
        # many short chats with a small model: one key head to each query head, heads of 64, OCP MXFP4, small pages
        {"name": "attention_200x600", "kind": "attention", "fmt": "mxfp4_e8m0", "heads": 12, "kv_heads": 12, "head_dim": 64, "seqs": 200,
         "keys": 600, "page": 16, "rows": 1, "spare": 5},
        # a few rows of each sequence at once (a draft being verified), 70B-shaped heads, E4M3 scales
        {"name": "attention_16x4000_rows", "kind": "attention", "fmt": "amxfp4_e4m3", "heads": 64, "kv_heads": 8, "head_dim": 128,
         "seqs": 16, "keys": 4000, "page": 32, "rows": 4, "spare": 0},
        # one decoding step of 32 conversations: plan, write and attention
        {"name": "step_32x4096", "kind": "step", "fmt": "amxfp4_e5m2", "heads": 32, "kv_heads": 8, "head_dim": 128, "seqs": 32,
         "keys": 4096, "page": 64, "rows": 1, "spare": 0, "short": False},
        # a step with drafts of up to six tokens, symmetric scales, one slot in ten idle, and rows to spare
        {"name": "step_48x2000_rows", "kind": "step", "fmt": "mxfp4_e5m2", "heads": 32, "kv_heads": 32, "head_dim": 128, "seqs": 48,
         "keys": 2000, "page": 32, "rows": 6, "spare": 9, "short": False},
    ]


HEADS = [(32, 8, 128), (64, 8, 128), (32, 32, 128), (40, 8, 128), (12, 12, 64), (32, 8, 64), (32, 4, 64)]


def _log_int(rng, lo, hi):
    return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))


def draw(rng):
    kind = rng.choices(["plan", "write", "attention", "step"], [2, 2, 5, 2])[0]
    page = rng.choice([16, 32, 64, 128, 256])
    if kind == "plan":
        seqs = _log_int(rng, 1, 1500)
        rows = _log_int(rng, 1, max(1, min(4000, 40000 // seqs)))
        keys = _log_int(rng, rows, max(rows, min(32768, 1000 * page)))
        return {"kind": kind, "seqs": seqs, "keys": keys, "page": page, "rows": rows, "spare": rng.choice([0, 1, 37]),
                "short": rng.random() < 0.3}
    heads, kv_heads, head_dim = rng.choice(HEADS)
    case = {"kind": kind, "fmt": rng.choice(list(FORMATS)), "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim}
    if kind == "write":
        seqs = _log_int(rng, 1, 300)
        rows = 1 if rng.random() < 0.5 else _log_int(rng, 1, max(1, 12000 // seqs))
        return {**case, "seqs": seqs, "keys": max(rows, _log_int(rng, 1, 2000)), "page": page, "rows": rows, "spare": rng.choice([0, 5])}
    rows = 1 if rng.random() < 0.6 else _log_int(rng, 1, 8)
    seqs = _log_int(rng, 1, 256)
    most = min(131072, int(1.0e9 / (seqs * kv_heads * head_dim)))  # what is read stays below the largest listed case
    if kind == "step":
        return {**case, "seqs": seqs, "keys": max(rows, _log_int(rng, 16, most // 2)), "page": page, "rows": rows,
                "spare": rng.choice([0, 3]), "short": rng.random() < 0.1}
    return {**case, "seqs": seqs, "keys": max(rows, _log_int(rng, 1, most)), "page": page, "rows": rows, "spare": rng.choice([0, 3])}


# ---- inputs ---------------------------------------------------------------------------------------------------------

def _lengths(case):
    """(tokens held, new rows) of each sequence. They go by the case, so that its work is known; the seed makes the values.
    plan and step: a few slots are idle (0 rows) or have ended (-1). attention: what is held counts the new rows."""
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    kind, keys, seqs = case["kind"], case["keys"], case["seqs"]
    held, new = [], []
    for _ in range(seqs):
        n = case["rows"] if case["rows"] == 1 or rng.random() < 0.3 else rng.randint(1, case["rows"])
        before = 0 if kind == "write" and case["rows"] > 8 else rng.randint(0, max(0, keys - n)) if rng.random() < 0.8 else max(0, keys - n)
        if kind in ("plan", "step") and seqs > 4:
            u = rng.random()
            n = -1 if u < 0.04 else 0 if u < 0.1 else n
        held.append(before)
        new.append(n)
    if seqs == 1:
        held[0] = keys - new[0]
    if kind in ("write", "attention"):
        held = [a + b for a, b in zip(held, new)]
    return held, new


def _rows(case):
    return sum(max(0, n) for n in _lengths(case)[1]) + case["spare"]


def _max_pages(case):
    return -(-case["keys"] // case["page"]) + 1


def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, device=DEV)


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _values(gen, rows, D, shift):
    """Keys or values of one head each: N(0, 1), a few outlier dimensions, some of them of one sign."""
    x = _randn(gen, rows, D)
    at = torch.randperm(D, generator=gen, device=DEV)
    x[:, at[:3]] *= 4.0
    x[:, at[3:D // 4]] += shift
    return x


def _pool(gen, case, pages):
    """Cache of `pages` pages whose rows are drawn from a bank of cast ones."""
    kind, asym = FORMATS[case["fmt"]]
    H, D, ps = case["kv_heads"], case["head_dim"], case["page"]
    pool = []
    for shift in (0.5, 1.0):
        codes, scales = _cast(_values(gen, 16384, D, shift), kind, asym)
        codes = codes[:, 0::2] | codes[:, 1::2] << 4
        at = torch.randint(0, 16384, (pages, H, ps), generator=gen, device=DEV)
        pool += [codes[at], scales[at].transpose(2, 3).contiguous()]
    return tuple(pool)


def _tables(gen, case, held, pages):
    """Block tables with pages in no order, and the ids that are left."""
    count = [-(-n // case["page"]) for n in held]
    ids = torch.randperm(pages, generator=gen, device=DEV).to(torch.int32)
    at = torch.arange(_max_pages(case), device=DEV)[None, :] < _ints(count)[:, None]
    table = torch.full((case["seqs"], _max_pages(case)), -1, dtype=torch.int32, device=DEV)
    table[at] = ids[:sum(count)]
    return table, ids[sum(count):]


def prepare(case, seed):
    gen = torch.Generator(DEV).manual_seed(seed)
    kind = case["kind"]
    held, new = _lengths(case)
    T, B = _rows(case), case["seqs"]
    s = {"case": case, "scratch": torch.empty(SCRATCH, dtype=torch.uint8, device=DEV)}
    used = sum(-(-n // case["page"]) for n in held)
    wanted = sum(-(-(h + n) // case["page"]) - -(-h // case["page"]) for h, n in zip(held, new) if n > 0)
    left = 0 if kind in ("write", "attention") else int(wanted * 0.8) if case["short"] else wanted + 7
    pages = used + left + 3
    s["table"], free = _tables(gen, case, held, pages)
    s["lens"], s["new_rows"] = _ints(held), _ints(new)
    if kind in ("plan", "step"):
        head = int(torch.randint(0, pages, (1,), generator=torch.Generator().manual_seed(seed)))
        s["queue"] = torch.full((pages,), -1, dtype=torch.int32, device=DEV)
        s["queue"][(head + torch.arange(left, device=DEV)) % pages] = free[:left]
        s["state"] = _ints([head, left, 0, 0])
        s["plan"] = tuple(torch.zeros(n, dtype=torch.int32, device=DEV) for n in (B, B + 1, T, T, 4))
    else:
        starts = [0]
        for n in new:
            starts.append(starts[-1] + n)
        at = [(b, held[b] - new[b] + i) for b in range(B) for i in range(new[b])]
        seq, pos = (torch.tensor(v, device=DEV) for v in zip(*at))
        s["starts"] = _ints(starts)
        s["positions"] = torch.full((T,), -1, dtype=torch.int32, device=DEV)
        s["positions"][:len(at)] = pos.int()
        s["slots"] = torch.full((T,), -1, dtype=torch.int32, device=DEV)
        s["slots"][:len(at)] = s["table"][seq, pos // case["page"]] * case["page"] + (pos % case["page"]).int()
    if kind == "plan":
        return s
    H, G, D = case["heads"], case["kv_heads"], case["head_dim"]
    s["scale"] = 1.0 / math.sqrt(D)
    if kind == "write":
        s["pool"] = tuple(torch.zeros((pages, G) + shape, dtype=torch.uint8, device=DEV) for shape in _shapes(case) * 2)
        s["k"], s["v"] = (torch.empty((T, G, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    else:
        s["pool"] = _pool(gen, case, pages)
        s["out"] = torch.zeros((T, H * D), dtype=torch.bfloat16, device=DEV)
    if kind == "attention":
        s["q"] = _randn(gen, T, H, D).to(torch.bfloat16)
    else:  # the output of the fused projection: queries | keys | values
        s["proj"] = torch.cat([_randn(gen, T, H * D)] + [torch.cat([_values(gen, T, D, x) for _ in range(G)], 1) for x in (0.5, 1.0)], 1)
        s["q"] = torch.zeros((T, H, D), dtype=torch.bfloat16, device=DEV)
    return s


def _shapes(case):
    D, ps = case["head_dim"], case["page"]
    return [(ps, D // 2), (D // 32, ps) + ((2,) if FORMATS[case["fmt"]][1] else ())]


# ---- one pass -------------------------------------------------------------------------------------------------------

@functools.lru_cache(None)
def _library(name):
    from paper_2411_09909_amd import binding
    if name is None:
        return binding, None
    kind, asym = FORMATS[name]
    return binding, binding.make_format({"e5m2": binding.FP8_E5M2, "e4m3": binding.FP8_E4M3, "e8m0": binding.E8M0_FLOOR}[kind], asym)


def run(s):
    case = s["case"]
    kind = case["kind"]
    binding, fmt = _library(case.get("fmt")) if own else (None, None)
    if kind in ("plan", "step"):
        if own:
            plan = binding.paged_plan(s["lens"], s["new_rows"], s["table"], s["queue"], s["state"], case["page"], out=s["plan"])
        else:
            plan = _plan(s)
        lens, starts, slots, positions, state = plan
        done = {"lens": lens, "starts": starts, "slots": slots, "positions": positions, "state": state, "table": s["table"],
                "queue": s["queue"]}
        if kind == "plan":
            return done
    else:
        lens, starts, slots, positions, done = s["lens"], s.get("starts"), s["slots"], s["positions"], {}
    q = s["q"]
    if kind in ("write", "step"):
        if own:
            binding.paged_write(fmt, s["proj"], s["pool"], slots, positions, case["heads"], THETA, q=q)
        else:
            _write(s, slots, positions)
        done["q"] = q
    if kind == "write":  # what the slots hold now, as values
        if own:
            binding.paged_read(fmt, s["pool"], slots, k=s["k"], v=s["v"])
        else:
            _read(s, slots)
        return {**done, "k": s["k"], "v": s["v"]}
    if own:
        out = binding.paged_attention(fmt, q, s["pool"], s["table"], lens, starts, positions, s["scale"], max_keys=case["keys"],
                                      out=s["out"], workspace=s["scratch"])
    else:
        out = _attention(s, q, lens, starts, positions)
    return {**done, "out": out}


def _plan(s):
    ps, queue, table = s["case"]["page"], s["queue"], s["table"]
    lens, new = s["lens"].long(), s["new_rows"].long()
    head, count = s["state"][0].long(), s["state"][1].long()
    B, width = table.shape
    pages, T = queue.numel(), s["plan"][2].numel()
    n = new.clamp(min=0)
    ends = n.cumsum(0)
    begins = ends - n
    held = (lens + ps - 1) // ps
    fits = (n > 0) & (lens + n <= width * ps) & (ends <= T)
    want = torch.where(fits, (lens + n + ps - 1) // ps - held, 0)
    upto = want.cumsum(0)
    ok = fits & ((want == 0) | (upto <= count))
    taken = torch.where(upto <= count, upto, 0).max()
    gone = new < 0
    back = torch.where(gone, held, 0)
    t = torch.arange(T, device=DEV)
    at = torch.searchsorted(ends, t, right=True)
    b = at.clamp(max=B - 1)
    live = (at < B) & ok[b]
    pos = torch.where(live, lens[b] + t - begins[b], -1)
    number = (pos // ps).clamp(min=0)
    fresh = number >= held[b]
    page = torch.where(fresh, queue[(head + upto[b] - want[b] + number - held[b]) % pages], table[b, number]).long()
    slots = torch.where(live, page * ps + pos % ps, -1)
    # entries for new pages and for the queue's end; what is not to be written goes behind the last element
    entries = torch.cat([table.reshape(-1), table.new_zeros(1)])
    entries[torch.where(live & fresh, b * width + number, B * width)] = page.int()
    p = torch.arange(width, device=DEV)[None, :]
    to = torch.where(gone[:, None] & (p < held[:, None]), (head + count + (back.cumsum(0) - back)[:, None] + p) % pages, pages)
    ring = torch.cat([queue, queue.new_zeros(1)])
    ring[to.reshape(-1)] = table.reshape(-1)
    table.copy_(entries[:-1].view(B, width))
    queue.copy_(ring[:-1])
    state = torch.stack([(head + taken) % pages, count - taken + back.sum(), ((n > 0) & ~ok).sum(), ends[-1].clamp(max=T)])
    starts = torch.cat([ends.new_zeros(1), ends]).clamp(max=T)
    lens = torch.where(gone, 0, torch.where(ok, lens + n, lens))
    return tuple(v.int() for v in (lens, starts, slots, pos, state))


def _cast(x, kind, asym):
    """x [.., D], BF16 values after rounding -> (codes [.., D], one to a byte; scales [.., D / 32(, 2)]), groups of 32."""
    x = x.to(torch.bfloat16).double()
    g = x.unflatten(-1, (-1, 32))
    most = [g.clamp(min=0).amax(-1), (-g).clamp(min=0).amax(-1)]
    if not asym:
        most = [torch.maximum(*most)]
    most = torch.stack(most, -1)
    if kind == "e8m0":  # the exponent, less that of the largest element
        scales = torch.where(most > 0, torch.frexp(most)[1] - 3 + 127, 0).clamp(min=0).to(torch.uint8)
    else:
        to, top = (torch.float8_e5m2, 57344.0) if kind == "e5m2" else (torch.float8_e4m3fn, 448.0)
        scales = (most / 6).clamp(max=top).float().to(to).view(torch.uint8)
    S = _scale_values(scales, kind).double()
    negative = torch.signbit(g)
    r = g.abs() / torch.where(negative, S[..., -1:], S[..., :1])
    # nearest of 0, .5, 1, 1.5, 2, 3, 4, 6; halfway cases to the even code; a scale of 0 (0 / 0 too) gives 0
    codes = sum((r >= m if even else r > m).to(torch.uint8) for m, even in
                ((0.25, 0), (0.75, 1), (1.25, 0), (1.75, 1), (2.5, 0), (3.5, 1), (5.0, 0)))
    codes = torch.where(r.isfinite(), codes, 0) + negative.to(torch.uint8) * 8
    return codes.to(torch.uint8).flatten(-2), scales if asym else scales[..., 0]


def _scale_values(scales, kind):
    if kind == "e8m0":
        return torch.where(scales > 0, scales.int() << 23, 1 << 22).view(torch.float32)  # the exponent's field; 2^-127 is subnormal
    return scales.view(torch.float8_e5m2 if kind == "e5m2" else torch.float8_e4m3fn).float()


def _grid():
    return torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], device=DEV)


def _dequantize(codes, scales, kind, asym):
    """codes [.., D / 2], scales [.., D / 32(, 2)] -> float32 [.., D]."""
    codes = codes.int()
    e = _grid()[torch.stack([codes & 15, codes >> 4], -1).flatten(-2)].unflatten(-1, (-1, 32))
    S = _scale_values(scales, kind)
    S = torch.where(torch.signbit(e), S[..., 1:], S[..., :1]) if asym else S[..., None]
    return (e * S).flatten(-2)


def _write(s, slots, positions):
    case = s["case"]
    kind, asym = FORMATS[case["fmt"]]
    H, G, D, ps = case["heads"], case["kv_heads"], case["head_dim"], case["page"]
    T = slots.numel()
    x = s["proj"].view(T, H + 2 * G, D)
    half = D // 2
    turn = positions.double()[:, None] * torch.exp(-math.log(THETA) * torch.arange(half, device=DEV, dtype=torch.float64) / half)
    cs, sn = turn.cos()[:, None], turn.sin()[:, None]
    a, b = x[:, :H + G, :half].double(), x[:, :H + G, half:].double()
    turned = torch.cat([a * cs - b * sn, b * cs + a * sn], -1).float().to(torch.bfloat16)
    live = (slots >= 0)
    s["q"].copy_(torch.where((positions >= 0)[:, None, None], turned[:, :H], s["q"]))
    # (rows without a slot write once more what the first row with one does; if there is none, what is there already)
    kc, ks, vc, vs = s["pool"]
    source = torch.where(live, torch.arange(T, device=DEV), live.int().argmax())
    slot = slots[source].clamp(min=0).long()
    page, at = slot // ps, slot % ps
    for y, codes, scales in ((turned[:, H:], kc, ks), (x[:, H + G:].to(torch.bfloat16), vc, vs)):
        c, sc = _cast(y, kind, asym)
        c = c[..., 0::2] | c[..., 1::2] << 4
        codes[page, :, at] = torch.where(live.any(), c[source], codes[page, :, at])
        scales[page, :, :, at] = torch.where(live.any(), sc[source], scales[page, :, :, at])


def _read(s, slots):
    kind, asym = FORMATS[s["case"]["fmt"]]
    ps = s["case"]["page"]
    kc, ks, vc, vs = s["pool"]
    live = slots >= 0
    slot = slots.clamp(min=0).long()
    page, at = slot // ps, slot % ps
    for codes, scales, to in ((kc, ks, s["k"]), (vc, vs, s["v"])):
        values = _dequantize(codes[page, :, at], scales[page, :, :, at], kind, asym)
        to.copy_(torch.where(live[:, None, None], values, 0))


def _attention(s, q, lens, starts, positions):
    case = s["case"]
    kind, asym = FORMATS[case["fmt"]]
    H, G, D, ps, B = case["heads"], case["kv_heads"], case["head_dim"], case["page"], case["seqs"]
    per, T, most = H // G, q.shape[0], case["rows"]
    table = s["table"][:, :-(-case["keys"] // ps)].clamp(min=0).long()
    L = table.shape[1] * ps
    kc, ks, vc, vs = s["pool"]

    def gathered(codes, scales):  # [B, G, L, D]
        c = codes[table].transpose(1, 2).reshape(B, G, L, D // 2)
        z = scales[table].transpose(1, 2).transpose(3, 4).reshape((B, G, L) + scales.shape[2:3] + scales.shape[4:])
        return _dequantize(c, z, kind, asym)

    # the rows of a sequence side by side: [B, most] row numbers, T for none
    row = starts[:-1, None].long() + torch.arange(most, device=DEV)[None, :]
    row = torch.where(row < starts[1:, None], row, T)
    pos = torch.cat([positions, positions.new_full((1,), -1)])[row]                # [B, most]
    q = torch.cat([q, q.new_zeros((1, H, D))])[row].float()                        # [B, most, H, D]
    q = q.view(B, most, G, per, D).permute(0, 2, 1, 3, 4).reshape(B, G, most * per, D)
    scores = (q @ gathered(kc, ks).transpose(2, 3)).view(B, G, most, per, L) * s["scale"]
    j = torch.arange(L, device=DEV)
    seen = (j <= pos[..., None]) & (j < lens[:, None, None])                       # [B, most, L]
    scores = scores.masked_fill(~seen[:, None, :, None], -math.inf)
    top = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - torch.where(top > -math.inf, top, 0.0))
    total = p.sum(-1, keepdim=True)
    p = p.view(B, G, most * per, L)
    o = (p @ gathered(vc, vs)).view(B, G, most, per, D)
    o = torch.where(total > 0, o / total, 0.0).permute(0, 2, 1, 3, 4).reshape(B, most, H * D)
    out = torch.cat([s["out"], s["out"].new_zeros((1, H * D))])
    out[row.reshape(-1)] = o.reshape(-1, H * D).to(torch.bfloat16)
    s["out"].copy_(out[:-1])
    return s["out"]


# ---- what a pass cannot do without ----------------------------------------------------------------------------------

def work(case):
    held, new = _lengths(case)
    kind, T, B, ps = case["kind"], _rows(case), case["seqs"], case["page"]
    rows = sum(max(0, n) for n in new)
    done = {"bytes": 0, "flops": 0}
    if kind in ("plan", "step"):
        taken = sum(-(-(h + n) // ps) - -(-h // ps) for h, n in zip(held, new) if n > 0)
        back = sum(-(-h // ps) for h, n in zip(held, new) if n < 0)
        done["bytes"] += 4 * (3 * B + B + 1 + 2 * T + 2 * (taken + back) + 8)
        if kind == "plan":
            return done
    H, G, D, pair = case["heads"], case["kv_heads"], case["head_dim"], 1 + FORMATS[case["fmt"]][1]
    token = 2 * G * (D // 2 + pair * D // 32)  # of the cache
    if kind in ("write", "step"):
        done["bytes"] += rows * (4 * (H + 2 * G) * D + 2 * H * D + token + 8)
        done["flops"] += rows * (H + G) * D * 3
    if kind == "write":
        done["bytes"] += rows * 4 * G * D
        return done
    if kind == "step":
        held = [h + n for h, n in zip(held, new)]
    seen = [h if n > 0 else 0 for h, n in zip(held, new)]
    done["bytes"] += sum(seen) * token + (0 if kind == "step" else 2 * rows * H * D) + 2 * rows * H * D
    done["bytes"] += sum(4 * -(-h // ps) for h in seen) + 4 * (2 * B + rows)
    done["flops"] += sum(4 * max(0, n) * h * H * D for h, n in zip(seen, new))
    return done


# ---- the same in 64 bits --------------------------------------------------------------------------------------------

def _power64(e):
    """2^e exactly (a library's pow need not be)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _scale64(byte, kind):
    """The number that a scale byte stands for, from its fields."""
    b = byte.long()
    if kind == "e8m0":
        return _power64(b - 127)
    m_bits, bias = (2, 15) if kind == "e5m2" else (3, 7)
    e, m = b >> m_bits, (b & ((1 << m_bits) - 1)).double() / (1 << m_bits)
    return torch.where(e > 0, (1 + m) * _power64(e - bias), m * 2.0 ** (1 - bias))


def _element64(code):
    m = (code & 7).long()
    size = torch.where(m < 4, m.double() / 2, torch.where(m == 7, 6.0, m.double() - 2))
    return torch.where(code >= 8, -size, size)


def _stored64(codes, scales, kind, asym):
    """codes [n, D / 2], scales [n, D / 32(, 2)] -> float64 [n, D]."""
    nibbles = torch.stack([codes % 16, codes // 16], 2).reshape(codes.shape[0], -1, 32)
    S = _scale64(scales, kind)
    return (_element64(nibbles) * (torch.where(nibbles >= 8, S[:, :, 1:], S[:, :, :1]) if asym else S[:, :, None])).reshape(codes.shape[0], -1)


def _cast64(x, kind, asym):
    """What the cast of x [n, D] (float64 holding BF16 values) stands for: the nearest representable values, by distance."""
    every = torch.arange(256 if kind == "e8m0" else 0x7C if kind == "e5m2" else 0x7F, device=DEV)
    table = _scale64(every, kind)
    grid = _element64(torch.arange(8, device=DEV))
    y = torch.zeros_like(x)
    for g in range(x.shape[1] // 32):
        v = x[:, 32 * g:32 * g + 32]
        for sign in (1, -1) if asym else (0,):
            member = v * sign > 0 if sign else v != 0
            top = torch.where(member, v.abs(), 0.0).amax(1)
            if kind == "e8m0":
                e = (top.view(torch.int64) >> 52) - 1023  # the floor of the logarithm
                S = torch.where(top > 0, _power64((e - 2).clamp(min=-127)), 0.0)
            else:
                S = table[_nearest(top / 6, table)]
            z = v.abs() / S.clamp(min=1e-300)[:, None]
            w = grid[_nearest(z, grid)] * S[:, None] * torch.sign(v)
            y[:, 32 * g:32 * g + 32] = torch.where(member, w, y[:, 32 * g:32 * g + 32])
    return y


def _nearest(x, sorted_values):
    """Index of the nearest of the values, the even one of two that are equally near."""
    hi = torch.searchsorted(sorted_values, x).clamp(1, sorted_values.numel() - 1)
    lo = hi - 1
    a, b = x - sorted_values[lo], sorted_values[hi] - x
    return torch.where((a < b) | ((a == b) & (lo % 2 == 0)), lo, hi)


def _turned64(x, pos):
    """x [n, heads, D] rotated by the positions, rounded to BF16 as a rotated head is."""
    half = x.shape[2] // 2
    inv = torch.pow(torch.tensor(THETA, dtype=torch.float64, device=DEV), -torch.arange(half, dtype=torch.float64, device=DEV) / half)
    z = torch.complex(x[..., :half], x[..., half:]) * torch.polar(torch.ones((), dtype=torch.float64, device=DEV), pos[:, None] * inv)[:, None]
    return torch.cat([z.real, z.imag], -1)


def _bf16(x):
    return x.float().to(torch.bfloat16).double()


def _stepped(case, s):
    """Lengths, row starts, positions and tables after the step, one sequence after the other (lists)."""
    ps, width = case["page"], s["table"].shape[1]
    table, queue = s["table"].tolist(), s["queue"].tolist()
    head, count = s["state"].tolist()[:2]
    T, pages = s["plan"][2].numel(), len(queue)
    lens, starts, positions, want_so_far = [], [0], [], 0
    for b, (h, n) in enumerate(zip(s["lens"].tolist(), s["new_rows"].tolist())):
        rows = max(n, 0)
        fits = rows > 0 and h + rows <= width * ps and starts[-1] + rows <= T
        first, want = -(-h // ps), 0
        if fits:
            want = -(-(h + rows) // ps) - first
            fits = want == 0 or want_so_far + want <= count
        if fits:
            for j in range(want):
                table[b][first + j] = queue[(head + want_so_far + j) % pages]
        want_so_far += want
        positions += [h + i if fits else -1 for i in range(rows)]
        lens.append(0 if n < 0 else h + rows if fits else h)
        starts.append(starts[-1] + rows)
    return lens, starts, positions, table


def exact(case, seed):
    kind = case["kind"]
    if kind == "plan":
        return None  # whole numbers
    s = prepare(case, seed)
    name, asym = FORMATS[case["fmt"]]
    H, G, D, ps = case["heads"], case["kv_heads"], case["head_dim"], case["page"]
    T = s["q"].shape[0]
    done = {}
    if kind == "step":
        lens, starts, positions, table = _stepped(case, s)
        done = {k: None for k in ("lens", "starts", "slots", "positions", "state", "table", "queue")}
    else:
        lens, starts, positions, table = (s[k].tolist() for k in ("lens", "starts", "positions", "table"))
    pos = torch.tensor((positions + [-1] * T)[:T], dtype=torch.float64, device=DEV)
    q = s["q"].double()
    if kind != "attention":
        x = s["proj"].double().view(T, H + 2 * G, D)
        live = (pos >= 0)[:, None, None]
        turned = _turned64(x[:, :H + G], pos)
        q = torch.where(live, turned[:, :H], 0.0)
        k = torch.where(live, _cast64(_bf16(turned[:, H:]).reshape(-1, D), name, asym).view(T, G, D), 0.0)
        v = torch.where(live, _cast64(_bf16(x[:, H + G:]).reshape(-1, D), name, asym).view(T, G, D), 0.0)
        done["q"] = q
        if kind == "write":
            return {**done, "k": k, "v": v}
        q = _bf16(q)
    out = torch.zeros((T, H, D), dtype=torch.float64, device=DEV)
    for b in range(case["seqs"]):
        rows = [t for t in range(starts[b], min(starts[b + 1], T)) if positions[t] >= 0]
        if not rows:
            continue
        ids = torch.tensor(table[b][:-(-lens[b] // ps)], device=DEV)
        at = pos[rows]
        for h in range(G):
            hold = []
            for codes, scales, fresh in ((s["pool"][0], s["pool"][1], 0), (s["pool"][2], s["pool"][3], 1)):
                hold.append(_stored64(codes[ids, h].reshape(-1, D // 2),
                                      scales[ids, h].transpose(1, 2).reshape((-1,) + scales.shape[2:3] + scales.shape[4:]), name, asym)[:lens[b]])
                if kind == "step":
                    hold[-1][at.long()] = (v if fresh else k)[rows, h]
            mine = q[rows][:, h * (H // G):(h + 1) * (H // G)]
            score = torch.einsum("rpd,jd->rpj", mine, hold[0]) * s["scale"]
            score.masked_fill_(torch.arange(lens[b], device=DEV)[None, None, :] > at[:, None, None], -math.inf)
            out[rows, h * (H // G):(h + 1) * (H // G)] = torch.softmax(score, -1) @ hold[1]
    return {**done, "out": out.view(T, H * D)}
