"""Scoring text with a quantized model, as cases that can be timed and compared: attention over packed documents, prompts with a
free prefix and windows, with capped scores and biases that fall with distance, the same for single new tokens over the paged
cache, and the log probabilities of tokens out of the logits.

    prompt       quantized attention (operands and probabilities cast to FP4) whose rows see a range of keys each
    decode       queries of new rows against what their sequences hold in the paged FP4 cache, scores capped or biased
    tokens       log probabilities of given tokens, entropy and the likeliest alternatives

    listed()              the named cases
    draw(rng)             one more case of the same ranges (rng: random.Random)
    prepare(case, seed)   the operands, masks, cache, logits and buffers that a program has in hand, on the GPU
    run(state)            one pass: plain torch where `own` is false, the library's calls where it is true
    work(case)            bytes and floating-point operations the pass cannot do without
    exact(case, seed)     the outputs in 64 bits
"""
import functools
import math
import random

import torch

own = False
DEV = "cuda"
SCRATCH = 256 << 20  # bytes of scratch memory that a program keeps

# name -> (scale format, sign-asymmetric); groups of 32
FORMATS = {
    "amxfp4_e5m2": ("e5m2", True),
    "mxfp4_e5m2": ("e5m2", False),
    "amxfp4_e4m3": ("e4m3", True),
    "amxfp4_e8m0": ("e8m0", True),
    "mxfp4_e8m0": ("e8m0", False),
}


def listed():
    return [
        # one short question, small model: launches and the latency of a few tiles
        {"name": "prompt_77", "kind": "prompt", "fmt": "amxfp4_e5m2", "heads": 12, "kv_heads": 12, "head_dim": 64, "rows": 77, "before": 0,
         "mask": "causal", "docs": 1, "empty": 0, "window": 0, "cap": 30.0, "slopes": False},
        # a window of evaluation text filled with short documents and some padding, capped scores
        {"name": "prompt_2048_documents", "kind": "prompt", "fmt": "amxfp4_e5m2", "heads": 32, "kv_heads": 8, "head_dim": 128, "rows": 2048,
         "before": 0, "mask": "documents", "docs": 9, "empty": 41, "window": 0, "cap": 50.0, "slopes": False},
        # one long document, scores that fall with distance instead of a rotary embedding
        {"name": "prompt_8192_distance", "kind": "prompt", "fmt": "amxfp4_e5m2", "heads": 32, "kv_heads": 8, "head_dim": 128, "rows": 8192,
         "before": 0, "mask": "causal", "docs": 1, "empty": 0, "window": 0, "cap": 0.0, "slopes": True},
        # questions whose prompts are read in both directions, answers from left to right; 70B-shaped heads, power-of-two scales
        {"name": "prompt_1504_prefixes", "kind": "prompt", "fmt": "amxfp4_e8m0", "heads": 64, "kv_heads": 8, "head_dim": 128, "rows": 1504,
         "before": 0, "mask": "prefix", "docs": 5, "empty": 0, "window": 0, "cap": 0.0, "slopes": False},
        # a chunk of a long prompt behind what is already there, layers of a window, heads of 64
        {"name": "prompt_1000_after_15000_window", "kind": "prompt", "fmt": "amxfp4_e4m3", "heads": 32, "kv_heads": 8, "head_dim": 64, "rows": 1000,
         "before": 15000, "mask": "window", "docs": 1, "empty": 0, "window": 4096, "cap": 50.0, "slopes": False},
        # the next token of one conversation
        {"name": "decode_1x700", "kind": "decode", "fmt": "amxfp4_e5m2", "heads": 32, "kv_heads": 8, "head_dim": 128, "seqs": 1, "keys": 700,
         "page": 64, "rows": 1, "spare": 0, "cap": 50.0, "slopes": False},
        # a batch of long conversations, capped scores
        {"name": "decode_48x12000", "kind": "decode", "fmt": "amxfp4_e5m2", "heads": 32, "kv_heads": 8, "head_dim": 128, "seqs": 48, "keys": 12000,
         "page": 64, "rows": 1, "spare": 0, "cap": 50.0, "slopes": False},
        # many chats with a small model whose scores fall with distance, drafts of a few rows
        {"name": "decode_150x900_rows", "kind": "decode", "fmt": "mxfp4_e8m0", "heads": 12, "kv_heads": 12, "head_dim": 64, "seqs": 150, "keys": 900,
         "page": 16, "rows": 3, "spare": 5, "cap": 0.0, "slopes": True},
        # the new token of one conversation and what else it could have been
        {"name": "tokens_1x128000_top20", "kind": "tokens", "rows": 1, "vocab": 128000, "dtype": "float32", "ld": 128000, "top": 20, "cap": 0.0,
         "ruled": 0, "missing": 0},
        # new tokens of a batch, an odd vocabulary with its rows close together, some of its ids ruled out
        {"name": "tokens_96x50001_top5", "kind": "tokens", "rows": 96, "vocab": 50001, "dtype": "bfloat16", "ld": 50001, "top": 5, "cap": 30.0,
         "ruled": 300, "missing": 0},
        # choices of a test scored: a large vocabulary, capped logits, whether the token is the likeliest one
        {"name": "tokens_700x256000_top1", "kind": "tokens", "rows": 700, "vocab": 256000, "dtype": "float32", "ld": 256000, "top": 1, "cap": 30.0,
         "ruled": 0, "missing": 200},
        # perplexity of a window of text, straight from the product's output
        {"name": "tokens_4096x128000", "kind": "tokens", "rows": 4096, "vocab": 128000, "dtype": "float32", "ld": 128064, "top": 10, "cap": 0.0,
         "ruled": 0, "missing": 9},
    ]


HEADS = [(32, 8, 128), (64, 8, 128), (32, 32, 128), (40, 8, 128), (12, 12, 64), (32, 8, 64), (32, 4, 64)]


def _log_int(rng, lo, hi):
    return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))


def draw(rng):
    kind = rng.choices(["prompt", "decode", "tokens"], [5, 3, 4])[0]
    cap = rng.choice([0.0, 30.0, 50.0, 15.5])
    if kind == "tokens":
        vocab = _log_int(rng, 1000, 260000)
        dtype = rng.choice(["float32", "bfloat16"])
        rows = _log_int(rng, 1, max(1, min(4096, 500_000_000 // vocab)))
        return {"kind": kind, "rows": rows, "vocab": vocab, "dtype": dtype, "ld": vocab + rng.choice([0, 0, 1, 24, 96]),
                "top": rng.choice([0, 1, 5, 20, 32]), "cap": cap, "ruled": rng.choice([0, 0, 100, vocab // 2]), "missing": rng.choice([0, rows // 3])}
    heads, kv_heads, head_dim = rng.choice(HEADS)
    case = {"kind": kind, "fmt": rng.choice(list(FORMATS)), "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim}
    slopes = rng.random() < 0.4
    if kind == "prompt":
        most = 1_000_000_000 // heads  # pairs of a row and a key to a head
        rows = _log_int(rng, 1, min(8192, int(math.sqrt(most))))
        mask = rng.choice(["causal", "documents", "prefix", "window"])
        before = 0 if mask in ("documents", "prefix") or rng.random() < 0.4 else _log_int(rng, 1, max(1, min(32000, most // rows - rows)))
        docs = _log_int(rng, 1, max(1, rows // 8)) if mask in ("documents", "prefix") else 1
        window = _log_int(rng, 1, 8192) if mask == "window" else 0
        empty = rng.choice([0, rows // 9]) if mask in ("documents", "prefix") else 0
        return {**case, "rows": rows, "before": before, "mask": mask, "docs": docs, "empty": empty, "window": window, "cap": cap, "slopes": slopes}
    if cap == 0.0 and not slopes:
        cap = 50.0
    rows = 1 if rng.random() < 0.6 else _log_int(rng, 1, 8)
    seqs = _log_int(rng, 1, 256)
    most = min(131072, int(1.0e9 / (seqs * kv_heads * head_dim)))
    return {**case, "seqs": seqs, "keys": max(rows, _log_int(rng, 1, most)), "page": rng.choice([16, 32, 64, 128, 256]), "rows": rows,
            "spare": rng.choice([0, 3]), "cap": cap, "slopes": slopes}


# ---- inputs ---------------------------------------------------------------------------------------------------------

def _rng(case):
    """Lengths go by the case, so that its work is known; the seed makes the values."""
    return random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))


def _ranges(case):
    """(first, last) key that each row of a prompt sees; last < first where it sees none."""
    rows, before = case["rows"], case["before"]
    if case["mask"] in ("causal", "window"):
        window = case["window"] or before + rows
        return [(max(0, before + i - window + 1), before + i) for i in range(rows)]
    rng = _rng(case)
    used = rows - case["empty"]
    ends = sorted(rng.sample(range(1, used), min(case["docs"], used) - 1)) + [used]
    seen, start = [], 0
    for end in ends:
        free = start + int((end - start) * rng.uniform(0.3, 0.7)) - 1 if case["mask"] == "prefix" else 0
        seen += [(start, max(i, free)) for i in range(start, end)]
        start = end
    return seen + [(0, -1)] * case["empty"]


def _lengths(case):
    """(tokens held with the new rows, new rows) of each sequence."""
    rng, keys = _rng(case), case["keys"]
    held, new = [], []
    for _ in range(case["seqs"]):
        n = case["rows"] if case["rows"] == 1 or rng.random() < 0.3 else rng.randint(1, case["rows"])
        before = rng.randint(0, max(0, keys - n)) if rng.random() < 0.8 else max(0, keys - n)
        held.append(before + n)
        new.append(n)
    if case["seqs"] == 1:
        held[0] = keys
    return held, new


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _values(gen, rows, D, shift):
    """Rows of queries, keys or values: N(0, 1), a few outlier dimensions, some of them of one sign."""
    x = torch.randn((rows, D), generator=gen, device=DEV)
    at = torch.randperm(D, generator=gen, device=DEV)
    x[:, at[:3]] *= 4.0
    x[:, at[3:D // 4]] += shift
    return x


def _packed(codes):
    return codes[..., 0::2] | codes[..., 1::2] << 4


def _slopes(case):
    H = case["heads"]
    return torch.exp2(-8.0 * torch.arange(1, H + 1, dtype=torch.float64) / H).float().to(DEV) if case["slopes"] else None


def prepare(case, seed):
    gen = torch.Generator(DEV).manual_seed(seed)
    s = {"case": case}
    if case["kind"] == "tokens":
        return _prepare_tokens(s, gen)
    s["scratch"] = torch.empty(SCRATCH, dtype=torch.uint8, device=DEV)
    s["scale"], s["slopes"] = 1.0 / math.sqrt(case["head_dim"]), _slopes(case)
    return _prepare_prompt(s, gen) if case["kind"] == "prompt" else _prepare_decode(s, gen)


def _prepare_prompt(s, gen):
    case = s["case"]
    kind, asym = FORMATS[case["fmt"]]
    H, G, D, Sq = case["heads"], case["kv_heads"], case["head_dim"], case["rows"]
    Sk = -(-(case["before"] + Sq) // 32) * 32
    for name, heads, rows, shift in (("q", H, Sq, 0.3), ("k", G, Sk, 0.5), ("v", G, Sk, 1.0)):
        x = _values(gen, heads * rows, D, shift).view(heads, rows, D)
        codes, scales = _cast(x.transpose(1, 2) if name == "v" else x, kind, asym)
        s[name] = _packed(codes).contiguous(), scales.contiguous()
    if case["mask"] == "causal":
        s["first"] = s["last"] = None
    else:
        seen = _ranges(case)
        s["first"] = _ints([a for a, _ in seen])
        s["last"] = _ints([b for _, b in seen]) if case["mask"] == "prefix" or case["empty"] else None
    s["out"] = torch.zeros((Sq, H * D), dtype=torch.bfloat16, device=DEV)
    return s


def _prepare_decode(s, gen):
    case = s["case"]
    kind, asym = FORMATS[case["fmt"]]
    H, G, D, ps, B = case["heads"], case["kv_heads"], case["head_dim"], case["page"], case["seqs"]
    held, new = _lengths(case)
    T = sum(new) + case["spare"]
    count = [-(-n // ps) for n in held]
    pages = sum(count) + 3
    width = -(-case["keys"] // ps) + 1
    # tables with pages in no order
    at = torch.arange(width, device=DEV)[None, :] < _ints(count)[:, None]
    s["table"] = torch.full((B, width), -1, dtype=torch.int32, device=DEV)
    s["table"][at] = torch.randperm(pages, generator=gen, device=DEV).to(torch.int32)[:sum(count)]
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    s["lens"], s["starts"] = _ints(held), _ints(starts)
    s["positions"] = _ints([held[b] - new[b] + i for b in range(B) for i in range(new[b])] + [-1] * case["spare"])
    # rows drawn from a bank of cast ones
    pool = []
    for shift in (0.5, 1.0):
        codes, scales = _cast(_values(gen, 16384, D, shift), kind, asym)
        at = torch.randint(0, 16384, (pages, G, ps), generator=gen, device=DEV)
        pool += [_packed(codes)[at], scales[at].transpose(2, 3).contiguous()]
    s["pool"] = tuple(pool)
    s["q"] = torch.randn((T, H, D), generator=gen, device=DEV).to(torch.bfloat16)
    s["out"] = torch.zeros((T, H * D), dtype=torch.bfloat16, device=DEV)
    return s


def _prepare_tokens(s, gen):
    case = s["case"]
    T, V = case["rows"], case["vocab"]
    wide = torch.empty((T, case["ld"]), dtype=getattr(torch, case["dtype"]), device=DEV)
    s["logits"] = wide[:, :V]
    s["logits"].normal_(0.0, 2.5, generator=gen)
    if case["ld"] > V:
        wide[:, V:] = math.nan  # not part of a row
    # a few candidates, each another token, stand out in every row; half of the targets are among them
    at = (torch.randint(0, V, (T, 1), generator=gen, device=DEV) + torch.arange(24, device=DEV) * (V // 24)) % V
    up = torch.rand((T, 24), generator=gen, device=DEV) * 14.0
    s["logits"].scatter_(1, at, up.to(wide.dtype))
    if case["ruled"]:
        s["logits"][:, V - case["ruled"]:] = -math.inf
    some = torch.rand(T, generator=gen, device=DEV)
    target = torch.where(some < 0.5, at[:, 0], torch.randint(0, V, (T,), generator=gen, device=DEV)).int()
    gone = torch.randperm(T, generator=gen, device=DEV)[:case["missing"]]
    target[gone] = -1
    s["targets"] = target
    f = lambda *shape: torch.zeros(shape, dtype=torch.float32, device=DEV)  # noqa: E731
    s["out"] = (f(T), f(T), f(T, case["top"]), torch.zeros((T, case["top"]), dtype=torch.int32, device=DEV))
    s["scratch"] = torch.empty(16 << 20, dtype=torch.uint8, device=DEV)
    return s


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
    if kind == "tokens":
        if own:
            binding, _ = _library(None)
            got = binding.token_logprobs(s["logits"], s["targets"], top=case["top"], cap=case["cap"], out=s["out"], workspace=s["scratch"])
        else:
            got = _tokens(s)
        return dict(zip(("logprobs", "entropy", "top_logprobs", "top_ids"), got))
    if own:
        binding, fmt = _library(case["fmt"])
        if kind == "prompt":
            return binding.attention_masked(fmt, *s["q"], *s["k"], *s["v"], s["scale"], cap=case["cap"], slopes=s["slopes"], first=s["first"],
                                            last=s["last"], causal=s["last"] is None, pos0=case["before"], out=s["out"], workspace=s["scratch"])
        return binding.paged_attention(fmt, s["q"], s["pool"], s["table"], s["lens"], s["starts"], s["positions"], s["scale"],
                                       max_keys=case["keys"], out=s["out"], workspace=s["scratch"], cap=case["cap"], slopes=s["slopes"])
    return _prompt(s) if kind == "prompt" else _decode(s)


def _cast(x, kind, asym):
    """x [.., K] -> (codes [.., K], one to a byte; scales [.., K / 32(, 2)]) of its BF16 values, groups of 32."""
    g = x.to(torch.bfloat16).float().unflatten(-1, (-1, 32))
    most = [g.clamp(min=0).amax(-1), (-g).clamp(min=0).amax(-1)]
    scales = _scale_bytes(torch.stack(most, -1) if asym else torch.maximum(*most)[..., None], kind)
    S = _scale_values(scales, kind).double()
    negative = torch.signbit(g)
    codes = _codes(g.double().abs() / torch.where(negative, S[..., -1:], S[..., :1])) + negative.to(torch.uint8) * 8
    return codes.flatten(-2), scales if asym else scales[..., 0]


def _scale_bytes(most, kind):
    """Scale bytes of groups from their largest magnitudes."""
    if kind == "e8m0":  # the exponent, less that of the largest element
        return torch.where(most > 0, torch.frexp(most)[1] - 3 + 127, 0).clamp(min=0).to(torch.uint8)
    to, top = (torch.float8_e5m2, 57344.0) if kind == "e5m2" else (torch.float8_e4m3fn, 448.0)
    return (most.double() / 6).clamp(max=top).float().to(to).view(torch.uint8)


def _codes(r):
    """Nearest of 0, .5, 1, 1.5, 2, 3, 4, 6; halfway cases to the even code; a scale of 0 (0 / 0 too) gives 0."""
    codes = sum((r >= m if even else r > m).to(torch.uint8) for m, even in
                ((0.25, 0), (0.75, 1), (1.25, 0), (1.75, 1), (2.5, 0), (3.5, 1), (5.0, 0)))
    return torch.where(r.isfinite(), codes, 0).to(torch.uint8)


def _scale_values(scales, kind):
    if kind == "e8m0":
        return torch.where(scales > 0, scales.int() << 23, 1 << 22).view(torch.float32)  # the exponent's field; 2^-127 is subnormal
    return scales.view(torch.float8_e5m2 if kind == "e5m2" else torch.float8_e4m3fn).float()


def _grid():
    return torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], device=DEV)


def _dequantize(codes, scales, kind, asym):
    """codes [.., K / 2], scales [.., K / 32(, 2)] -> float32 [.., K]."""
    codes = codes.int()
    e = _grid()[torch.stack([codes & 15, codes >> 4], -1).flatten(-2)].unflatten(-1, (-1, 32))
    S = _scale_values(scales, kind)
    S = torch.where(torch.signbit(e), S[..., 1:], S[..., :1]) if asym else S[..., None]
    return (e * S).flatten(-2)


def _scored(scores, case, slopes, distance):
    """Capped, and less the slope of the head for each key of distance. scores [.., H, rows, keys]"""
    if case["cap"]:
        scores = torch.tanh(scores / case["cap"]) * case["cap"]
    return scores if slopes is None else scores - slopes[:, None, None] * distance


def _prompt(s):
    case = s["case"]
    kind, asym = FORMATS[case["fmt"]]
    H, G, D, Sq = case["heads"], case["kv_heads"], case["head_dim"], case["rows"]
    q, k, v = (_dequantize(*s[n], kind, asym) for n in ("q", "k", "v"))        # [H, Sq, D], [G, Sk, D], [G, D, Sk]
    Sk = k.shape[1]
    at = case["before"] + torch.arange(Sq, device=DEV)[:, None]
    j = torch.arange(Sk, device=DEV)
    scores = (q.view(G, -1, D) @ k.transpose(1, 2)).view(H, Sq, Sk) * s["scale"]
    scores = _scored(scores, case, s["slopes"], (at - j).abs().float())
    seen = j <= (at if s["last"] is None else s["last"][:, None])
    if s["first"] is not None:
        seen = seen & (j >= s["first"][:, None])
    x = scores.masked_fill_(~seen, -math.inf).view(H, Sq, Sk // 32, 32)
    tops = x.amax(-1).cummax(-1).values                                       # the running maximum, tile by tile
    top = tops[..., -1:]
    p = torch.exp(x - torch.where(tops > -math.inf, tops, 0.0)[..., None])
    late = torch.exp(tops - torch.where(top > -math.inf, top, 0.0))           # what comes of a tile's weights at the end
    total = (p.sum(-1) * late).sum(-1, keepdim=True)
    S = _scale_values(_scale_bytes(p.amax(-1), kind), kind)
    p = _grid()[_codes(p / S[..., None]).int()] * (S * late)[..., None]       # each tile's 32 weights cast as one group
    o = (p.view(G, -1, Sk) @ v.transpose(1, 2).contiguous()).view(H, Sq, D)
    o = torch.where(total > 0, o / total, 0.0)
    s["out"].copy_(o.transpose(0, 1).reshape(Sq, H * D))
    return s["out"]


def _decode(s):
    case = s["case"]
    kind, asym = FORMATS[case["fmt"]]
    H, G, D, ps, B = case["heads"], case["kv_heads"], case["head_dim"], case["page"], case["seqs"]
    lens, starts, positions, q = s["lens"], s["starts"], s["positions"], s["q"]
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
    q = q.view(B, most, G, per, D).permute(0, 2, 3, 1, 4).reshape(B, G, per * most, D)
    scores = (q @ gathered(kc, ks).transpose(2, 3)).view(B, H, most, L) * s["scale"]
    j = torch.arange(L, device=DEV)
    scores = _scored(scores, case, s["slopes"], (pos[:, None, :, None] - j).abs().float())
    seen = (j <= pos[..., None]) & (j < lens[:, None, None])                       # [B, most, L]
    scores = scores.masked_fill(~seen[:, None], -math.inf)
    top = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - torch.where(top > -math.inf, top, 0.0))
    total = p.sum(-1, keepdim=True)
    o = (p.view(B, G, per * most, L) @ gathered(vc, vs)).view(B, H, most, D)
    o = torch.where(total > 0, o / total, 0.0).transpose(1, 2).reshape(B, most, H * D)
    out = torch.cat([s["out"], s["out"].new_zeros((1, H * D))])
    out[row.reshape(-1)] = o.reshape(-1, H * D).to(torch.bfloat16)
    s["out"].copy_(out[:-1])
    return s["out"]


def _tokens(s):
    case = s["case"]
    T, V = s["logits"].shape
    x = s["logits"].float()
    if case["cap"]:  # (what is ruled out stays so)
        x = torch.where(x > -math.inf, torch.tanh(x / case["cap"]) * case["cap"], x)
    top = x.amax(1, keepdim=True)
    e = torch.exp(x - top)
    total = e.sum(1, keepdim=True)
    lse = top + torch.log(total)
    mean = (e * torch.where(e > 0, x - top, 0.0)).sum(1) / total[:, 0]
    logprob = x.gather(1, s["targets"].clamp(min=0).long()[:, None])[:, 0] - lse[:, 0]
    logprob = torch.where(s["targets"] >= 0, logprob, 0.0)
    # by the logits as they are: their bits as integers in the same order, and of equal ones the lowest id first
    bits = (s["logits"].float() + 0.0).view(torch.int32)
    order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long() << 32 | (V - 1 - torch.arange(V, device=DEV))
    ids = V - 1 - (order.topk(case["top"], 1).values & 0xFFFFFFFF)
    return logprob, torch.log(total[:, 0]) - mean, x.gather(1, ids) - lse, ids.int()


# ---- what a pass cannot do without ----------------------------------------------------------------------------------

def work(case):
    if case["kind"] == "tokens":
        T, V, size = case["rows"], case["vocab"], 4 if case["dtype"] == "float32" else 2
        return {"bytes": T * V * size + T * (12 + 8 * case["top"]), "flops": T * V * (5 if not case["cap"] else 10)}
    H, G, D, pair = case["heads"], case["kv_heads"], case["head_dim"], 1 + FORMATS[case["fmt"]][1]
    row = D // 2 + pair * D // 32
    if case["kind"] == "prompt":
        Sq, keys = case["rows"], case["before"] + case["rows"]
        seen = _ranges(case)
        least = min((a for a, b in seen if b >= a), default=0)
        return {"bytes": Sq * H * (row + 2 * D) + 2 * (keys - least) * G * row + (0 if case["mask"] == "causal" else 4 * Sq),
                "flops": 4 * D * H * sum(max(0, b - a + 1) for a, b in seen)}
    held, new = _lengths(case)
    T = sum(new)
    return {"bytes": sum(held) * 2 * G * row + 4 * T * H * D + sum(4 * -(-h // case["page"]) for h in held) + 4 * (2 * len(held) + T),
            "flops": sum(4 * n * (h - (n - 1) // 2) * H * D for h, n in zip(held, new))}


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
    """codes [n, K / 2], scales [n, K / 32(, 2)] -> float64 [n, K]."""
    nibbles = torch.stack([codes % 16, codes // 16], 2).reshape(codes.shape[0], -1, 32)
    S = _scale64(scales, kind)
    return (_element64(nibbles) * (torch.where(nibbles >= 8, S[:, :, 1:], S[:, :, :1]) if asym else S[:, :, None])).reshape(codes.shape[0], -1)


def _nearest(x, sorted_values):
    """Index of the nearest of the values, the even one of two that are equally near."""
    hi = torch.searchsorted(sorted_values, x).clamp(1, sorted_values.numel() - 1)
    lo = hi - 1
    a, b = x - sorted_values[lo], sorted_values[hi] - x
    return torch.where((a < b) | ((a == b) & (lo % 2 == 0)), lo, hi)


def _weights64(p, kind):
    """What the cast of weights p [rows, 32] in 0 .. 1 stands for."""
    top = p.amax(1)
    if kind == "e8m0":
        e = (top.view(torch.int64) >> 52) - 1023  # the floor of the logarithm
        S = torch.where(top > 0, _power64((e - 2).clamp(min=-127)), 0.0)
    else:
        table = _scale64(torch.arange(0x7C if kind == "e5m2" else 0x7F, device=DEV), kind)
        S = table[_nearest(top / 6, table)]
    grid = _element64(torch.arange(8, device=DEV))
    w = grid[_nearest((p / S.clamp(min=1e-300)[:, None]).contiguous(), grid)] * S[:, None]
    return torch.where(p > 0, w, 0.0)


def _scores64(case, q, k, at, slope, scale):
    """q [n, D], k [m, D] at positions 0 .. m - 1, rows at `at`."""
    s = (q @ k.T) * scale
    if case["cap"]:
        s = case["cap"] * (s / case["cap"]).tanh()
    if slope is not None:
        s = s - float(slope) * (at[:, None] - torch.arange(k.shape[0], device=DEV, dtype=torch.float64)).abs()
    return s


def exact(case, seed):
    s = prepare(case, seed)
    return {"prompt": _prompt64, "decode": _decode64, "tokens": _tokens64}[case["kind"]](case, s)


def _prompt64(case, s):
    kind, asym = FORMATS[case["fmt"]]
    H, G, D, Sq = case["heads"], case["kv_heads"], case["head_dim"], case["rows"]
    Sk = s["k"][0].shape[1]
    seen = torch.tensor(_ranges(case), device=DEV)
    out = torch.zeros((Sq, H, D), dtype=torch.float64, device=DEV)
    at = torch.arange(Sq, device=DEV, dtype=torch.float64) + case["before"]
    for h in range(H):
        g = h // (H // G)
        q, k, v = (_stored64(s[n][0][i], s[n][1][i], kind, asym) for n, i in (("q", h), ("k", g), ("v", g)))
        slope = None if s["slopes"] is None else s["slopes"][h].item()
        x = _scores64(case, q, k, at, slope, s["scale"])
        j = torch.arange(Sk, device=DEV)
        x[(j < seen[:, :1]) | (j > seen[:, 1:])] = -math.inf
        m = torch.full((Sq,), -math.inf, dtype=torch.float64, device=DEV)
        total, o = torch.zeros_like(m), torch.zeros((Sq, D), dtype=torch.float64, device=DEV)
        for t in range(0, Sk, 32):  # the recurrence, tile by tile, for the rows that see any of its keys
            rows = ((seen[:, 0] < t + 32) & (seen[:, 1] >= t) & (seen[:, 1] >= seen[:, 0])).nonzero()[:, 0]
            if not rows.numel():
                continue
            tile = x[rows, t:t + 32]
            new = torch.maximum(m[rows], tile.amax(1))
            p, keep = torch.exp(tile - new[:, None]), torch.exp(m[rows] - new)
            total[rows] = total[rows] * keep + p.sum(1)
            o[rows] = o[rows] * keep[:, None] + _weights64(p, kind) @ v[:, t:t + 32].T
            m[rows] = new
        out[:, h] = torch.where(total[:, None] > 0, o / total[:, None], 0.0)
    return out.view(Sq, H * D)


def _decode64(case, s):
    name, asym = FORMATS[case["fmt"]]
    H, G, D, ps = case["heads"], case["kv_heads"], case["head_dim"], case["page"]
    held, new = _lengths(case)
    out = torch.zeros((s["q"].shape[0], H, D), dtype=torch.float64, device=DEV)
    first = 0
    for b, (n, rows) in enumerate(zip(held, new)):
        ids = s["table"][b][:-(-n // ps)].long()
        at = torch.arange(n - rows, n, device=DEV, dtype=torch.float64)
        for g in range(G):
            k, v = (_stored64(c[ids, g].reshape(-1, D // 2), z[ids, g].transpose(1, 2).reshape((-1,) + z.shape[2:3] + z.shape[4:]), name, asym)[:n]
                    for c, z in (s["pool"][:2], s["pool"][2:]))
            for h in range(g * (H // G), (g + 1) * (H // G)):
                x = _scores64(case, s["q"][first:first + rows, h].double(), k, at, None if s["slopes"] is None else s["slopes"][h].item(), s["scale"])
                x.masked_fill_(torch.arange(n, device=DEV)[None, :] > at[:, None], -math.inf)
                out[first:first + rows, h] = torch.softmax(x, -1) @ v
        first += rows
    return out.view(-1, H * D)


def _tokens64(case, s):
    T, V, top = case["rows"], case["vocab"], case["top"]
    logprobs, entropy = torch.zeros(2, T, dtype=torch.float64, device=DEV)
    tops = torch.zeros((T, top), dtype=torch.float64, device=DEV)
    for t in range(T):
        x = s["logits"][t].double()
        live = x > -math.inf
        y = case["cap"] * torch.tanh(x / case["cap"]) if case["cap"] else x
        y = torch.where(live, y, -math.inf)
        z = torch.log_softmax(y, 0)
        entropy[t] = -(z.exp()[live] * z[live]).sum()
        logprobs[t] = torch.where(s["targets"][t] >= 0, z[s["targets"][t].clamp(min=0).long()], 0.0)
        if top:
            tops[t] = z.topk(top).values
    return {"logprobs": logprobs, "entropy": entropy, "top_logprobs": tops, "top_ids": None}
