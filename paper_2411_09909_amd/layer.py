"""One LLaMA-style decoder layer (grouped-query attention, rotary embedding, gated MLP) whose seven matrix
multiplications all go through the quantized path: every operand is cast with amxfp4_quantize and multiplied with
amxfp4_gemm (Sec. 5.1: the linear projections and both attention products are quantized, the rest stays BF16).

This module only sequences library calls; the arithmetic is in libamxfp4 (binding.py marshals the arguments).
Shapes for a sequence of S tokens, H query heads, G key/value heads (H = G * per), head size D, model width W = H * D,
MLP width F:
  qkv    = cast(rmsnorm(x)) . Wqkv^T                  [S, W + 2 G D]
  scores = cast(rope(q)) . cast(rope(k))^T            batch G, [per * S, S]   (the `per` query heads that share a key
                                                                                head are stacked along the rows)
  o      = cast(softmax(scores)) . cast(v)^T          batch G, [per * S, D]   (P grouped along the keys, V cast down
                                                                                its columns)
  x2     = x + cast(merge(o)) . Wo^T
  out    = x2 + cast(silu(g) * u) . Wd^T,  (g | u) = cast(rmsnorm(x2)) . Wgu^T
With fused_attention=True the two attention products and the softmax between them are one call (binding.attention):
the attention map is not materialised and its tiles are cast relative to the running row maximum, which gives
slightly different numbers than casting the normalised map.
With score_cap, slopes or a range of keys for each row (packed documents, prefixes, windows) it is binding.attention_masked, and step() hands
cap and slopes on too. LMHead is what follows the last layer when text is scored: the normalisation, the product with the vocabulary's
weights and the log probabilities, a number of rows at a time.
step() is the same layer for sequences that are being served: their new rows, packed into one batch, against the keys and values
that a PagedCache holds. The queries and the probabilities stay BF16 there; keys and values are cast per token along D.
"""
import math
from dataclasses import dataclass

import torch

from . import binding


@dataclass
class LayerConfig:
    d_model: int = 4096
    n_heads: int = 32
    n_kv_heads: int = 8
    head_dim: int = 128
    d_ff: int = 14336
    eps: float = 1e-5
    rope_theta: float = 500000.0
    score_cap: float = 0.0  # attention scores s become score_cap tanh(s / score_cap); 0: as they are


WEIGHT_SHAPES = lambda c: {  # noqa: E731  (name -> [out features, in features])
    "wq": (c.n_heads * c.head_dim, c.d_model), "wk": (c.n_kv_heads * c.head_dim, c.d_model),
    "wv": (c.n_kv_heads * c.head_dim, c.d_model), "wo": (c.d_model, c.n_heads * c.head_dim),
    "wg": (c.d_ff, c.d_model), "wu": (c.d_ff, c.d_model), "wd": (c.d_model, c.d_ff)}


class PagedCache:
    """The FP4 keys and values of up to `seqs` sequences for `layers` layers, in pages of `page_size` tokens that the sequences share
    (a page has the same id in every layer), at most `max_keys` tokens, rounded up to whole pages, to a sequence. All of it stays on the GPU: a step with plan()
    and DecoderLayer.step() waits for nothing and can be captured in a graph."""

    def __init__(self, cfg, fmt, seqs, pages, max_keys, page_size=64, layers=1, device="cuda"):
        self.page_size = page_size
        self.pools = [binding.paged_pool(fmt, pages, cfg.n_kv_heads, cfg.head_dim, page_size, device) for _ in range(layers)]
        self.table = torch.full((seqs, -(-max_keys // page_size)), -1, dtype=torch.int32, device=device)
        self.queue = torch.arange(pages, dtype=torch.int32, device=device)
        # lengths | queue head, free pages, refused, rows: one buffer, so that a step moves them on with one copy
        self._now = torch.zeros(seqs + 4, dtype=torch.int32, device=device)
        self._now[seqs + 1] = pages
        self.lens, self.state = self._now[:seqs], self._now[seqs:]

    def plan(self, new_rows, rows):
        """Pages and places for a step: new_rows int32 [seqs] on the GPU: how many of the batch's `rows` rows each sequence has, in its
        order; -1 ends a sequence and gives its pages back, 0 leaves it alone. One call to a step, for all layers. A sequence whose rows
        find no pages or no room is left as it was, and state[2] counts those: their rows have slot -1 and mean nothing behind step().
        A sequence does not shrink. To take back rows of a draft, keep copies of `lens` and `state` from before its plan, copy them back, and
        plan and store the accepted rows as if there had been no draft (they may come into other pages)."""
        after = torch.empty_like(self._now)
        out = (after[:self.lens.numel()], self.lens.new_empty(self.lens.numel() + 1), self.lens.new_empty(rows),
               self.lens.new_empty(rows), after[self.lens.numel():])
        plan = binding.paged_plan(self.lens, new_rows, self.table, self.queue, self.state, self.page_size, out=out)
        self._now.copy_(after)
        return plan


class DecoderLayer:
    """weights: dict name -> BF16 CUDA tensor (WEIGHT_SHAPES) plus "norm1" / "norm2" FP32 [d_model]. The weights are
    cast once here (they are static in inference); forward() casts the activations."""

    def __init__(self, cfg, weights, fmt, baseline=False, fused_attention=False, fused_glu=None, fused_norm=None,
                 fused_rope=None, prepared_weights=False, slopes=None):
        """slopes: float32 [n_heads] on the GPU: scores of a head fall by so much for each key of distance (with or without a cap, these need
        fused_attention in forward()). They come beside the rotary embedding, which is always there."""
        self.cfg, self.fmt, self.baseline, self.fused_attention = cfg, fmt, baseline, fused_attention
        self.slopes = slopes
        # the rotary embedding casts its result (Q and K never exist as BF16 tensors): same bits
        if fused_rope is None:
            fused_rope = fmt.group_size == 32 and cfg.head_dim % 64 == 0 and cfg.head_dim <= 256
        self.fused_rope = fused_rope
        # the two normalisations cast their result in registers (and the second adds the residual first): same bits
        if fused_norm is None:
            fused_norm = fmt.group_size in (16, 32, 64) and cfg.d_model <= 16384
        self.fused_norm = fused_norm
        # the gate / up projection with the gated activation in its epilogue (the FP32 product is never written)
        if fused_glu is None:
            fused_glu = cfg.d_ff % 32 == 0
        self.fused_glu = fused_glu
        q = lambda w: binding.quantize(fmt, w.contiguous(), baseline=baseline)  # noqa: E731
        self.wqkv = q(torch.cat([weights["wq"], weights["wk"], weights["wv"]], 0))
        self.wo = q(weights["wo"])
        self.wgu = q(binding.interleave_gate_up(weights["wg"], weights["wu"]) if fused_glu
                     else torch.cat([weights["wg"], weights["wu"]], 0))
        self.wd = q(weights["wd"])
        self.norm1, self.norm2 = weights["norm1"].contiguous(), weights["norm2"].contiguous()
        self._ws = None
        # static weights: their kernel-private form written once (2 bytes per element of extra memory for the formats
        # that multiply on BF16 panels, nothing for the power-of-two formats); same bits
        self.prepared = None
        if prepared_weights and not baseline:
            self.prepared = {id(w): binding.prepare_weights(fmt, w[0], w[1])
                             for w in (self.wqkv, self.wo, self.wgu, self.wd)}

    def _workspace(self, need, device):
        """One buffer that grows for the layer's calls, which run one after another; a graph gets buffers of its own, so that what it
        was captured with neither goes away nor is another graph's too."""
        if torch.cuda.is_current_stream_capturing():
            return torch.empty(need, dtype=torch.uint8, device=device)
        if self._ws is None or self._ws.numel() < need:
            self._ws = torch.empty(need, dtype=torch.uint8, device=device)
        return self._ws

    def _gemm(self, a, b):
        fmt = self.fmt
        batch = a[0].shape[0] if a[0].dim() == 3 else 1
        need = binding.gemm_workspace_bytes(fmt, a[0].shape[-2], b[0].shape[-2], a[0].shape[-1] * 2, batch)
        ws = self._workspace(need, a[0].device) if need else None
        if self.prepared is not None and id(b) in self.prepared and batch == 1:
            return binding.gemm_prepared(fmt, a[0], a[1], b[0], b[1], self.prepared[id(b)], workspace=ws)
        return binding.gemm(fmt, a[0], a[1], b[0], b[1], workspace=ws, baseline=self.baseline)

    def _plain_fmt(self):
        """the format for the entry points that have no mxfp4_* twin: symmetric when this layer is the baseline"""
        return binding.make_format(self.fmt.scale, False, self.fmt.group_size) if self.baseline else self.fmt

    def _cast(self, x, k_axis=-1):
        return binding.quantize(self.fmt, x, k_axis=k_axis, baseline=self.baseline)

    def forward(self, x, pos0=0, first=None, last=None):
        """x BF16 [rows, d_model], rows a multiple of 32, the first at position pos0. first, last: int32 [rows] on the GPU: the first and the last of
        these rows that each of them sees, as binding.attention_masked() takes them (last instead of the causal mask: none behind the row
        itself is kept from it then); they need fused_attention. step() knows no such ranges: its rows see all that their sequence holds up to them."""
        c = self.cfg
        masked = first is not None or last is not None or c.score_cap or self.slopes is not None
        if masked and not self.fused_attention:
            raise binding.AmxError("forward: ranges of keys, score_cap and slopes need fused_attention")
        S, G, D = x.shape[0], c.n_kv_heads, c.head_dim
        per = c.n_heads // G
        nsc = self.wqkv[1].shape[2:]  # () or (2,): scale entries per group

        qkv = self._qkv(x)
        v = binding.split_heads_rope(qkv, (c.n_heads + G) * D, G, D, False)
        if self.fused_rope:
            # rotary embedding and the cast of Q and K along the head dimension in one launch each (same bits)
            qc, qs = binding.split_heads_rope_quantize(self._plain_fmt(), qkv, 0, c.n_heads, D, pos0, c.rope_theta)
            kc, ks = binding.split_heads_rope_quantize(self._plain_fmt(), qkv, c.n_heads * D, G, D, pos0, c.rope_theta)
        else:
            q = binding.split_heads_rope(qkv, 0, c.n_heads, D, True, pos0, c.rope_theta)
            k = binding.split_heads_rope(qkv, c.n_heads * D, G, D, True, pos0, c.rope_theta)
            qc, qs = self._cast(q.view(c.n_heads * S, D))
            kc, ks = self._cast(k.view(G * S, D))
        if self.fused_attention:
            vc, vs = self._cast_v(v, nsc)
            fmt = binding.make_format(self.fmt.scale, False, 32) if self.baseline else self.fmt
            if masked:
                need = binding.attention_masked_workspace_bytes(fmt, c.n_heads, G, S, S, D)
                o = binding.attention_masked(fmt, qc.view(c.n_heads, S, D // 2), qs.view(c.n_heads, S, D // 32, *nsc), kc.view(G, S, D // 2),
                                             ks.view(G, S, D // 32, *nsc), vc, vs, 1.0 / math.sqrt(D), causal=last is None, first=first, last=last,
                                             cap=c.score_cap, slopes=self.slopes, workspace=self._workspace(need, x.device),
                                             out=torch.empty((S, c.n_heads * D), dtype=torch.bfloat16, device=x.device))
                return self._after_attention(x, o)
            need = binding.attention_workspace_bytes(fmt, c.n_heads, G, S, S, D)
            # (the kernel writes its output merged and in BF16: what merge_heads would make of the FP32 result)
            o = binding.attention(fmt, qc.view(c.n_heads, S, D // 2), qs.view(c.n_heads, S, D // 32, *nsc),
                                  kc.view(G, S, D // 2), ks.view(G, S, D // 32, *nsc), vc, vs, 1.0 / math.sqrt(D),
                                  True, workspace=self._workspace(need, x.device), merged=True)
            return self._after_attention(x, o)
        scores = self._gemm((qc.view(G, per * S, D // 2), qs.view(G, per * S, D // 32, *nsc)),
                            (kc.view(G, S, D // 2), ks.view(G, S, D // 32, *nsc)))
        p = binding.softmax_causal(scores, 1.0 / math.sqrt(D))
        del scores
        pc, ps = self._cast(p.view(G * per * S, S))
        del p
        vc, vs = self._cast_v(v, nsc)
        o = self._gemm((pc.view(G, per * S, S // 2), ps.view(G, per * S, S // 32, *nsc)), (vc, vs))
        return self._after_attention(x, binding.merge_heads(o, G, per, S, D))

    def _qkv(self, x):
        if self.fused_norm:
            return self._gemm(binding.rmsnorm_quantize(self._plain_fmt(), x, self.norm1, self.cfg.eps), self.wqkv)
        return self._gemm(self._cast(binding.rmsnorm(x, self.norm1, self.cfg.eps)), self.wqkv)

    def step(self, x, cache, plan, layer=0, max_keys=0):
        """x BF16 [rows, d_model]: the new rows of the cache's sequences, packed as in the `plan` that cache.plan() made for them (single
        tokens, chunks of prompts or both). Stores their keys and values in pool `layer` of the cache, which is kept in the layer's
        format (symmetric for the baseline), and returns the layer's output [rows, d_model]. Rows of refused sequences and behind the
        last sequence come out without a meaning. max_keys: as for binding.paged_attention(). The layer's calls take turns on one stream, as in forward()."""
        c = self.cfg
        fmt, pool = self._plain_fmt(), cache.pools[layer]
        rows = x.shape[0]
        if pool.k_codes.shape[1] != c.n_kv_heads or pool.k_codes.shape[3] * 2 != c.head_dim:  # (a narrower one would take the wrong columns)
            raise binding.AmxError("step: a cache of %d key heads of %d, the layer has %d of %d" % (
                pool.k_codes.shape[1], pool.k_codes.shape[3] * 2, c.n_kv_heads, c.head_dim))
        q = torch.empty((rows, c.n_heads, c.head_dim), dtype=torch.bfloat16, device=x.device)
        binding.paged_write(fmt, self._qkv(x), pool, plan.slots, plan.positions, c.n_heads, c.rope_theta, q=q)
        need = binding.paged_attention_workspace_bytes(fmt, pool, rows, c.n_heads, cache.lens.numel(), max_keys)
        attn = torch.empty((rows, c.n_heads * c.head_dim), dtype=torch.bfloat16, device=x.device)
        binding.paged_attention(fmt, q, pool, cache.table, plan.lens, plan.starts, plan.positions, 1.0 / math.sqrt(c.head_dim), max_keys,
                                out=attn, workspace=self._workspace(need, x.device), cap=c.score_cap, slopes=self.slopes)
        return self._after_attention(x, attn)

    def _cast_v(self, v, nsc):
        G, S, D = v.shape
        vc = torch.empty((G, D, S // 2), dtype=torch.uint8, device=v.device)
        vs = torch.empty((G, D, S // 32) + tuple(nsc), dtype=torch.uint8, device=v.device)
        # V of one head is [S, D]; its groups run down the columns (along the keys); all heads in one launch
        fmt = binding.make_format(self.fmt.scale, False, self.fmt.group_size) if self.baseline else self.fmt
        binding.quantize_batched(fmt, v, k_axis=1, codes=vc, scales=vs)
        return vc, vs

    def _after_attention(self, x, attn):
        c = self.cfg
        if self.fused_norm:
            x2, *hc = binding.rmsnorm_quantize(self._plain_fmt(), x, self.norm2, c.eps,
                                               y=self._gemm(self._cast(attn), self.wo))
        else:
            x2 = binding.residual_add(x, self._gemm(self._cast(attn), self.wo))
            hc = self._cast(binding.rmsnorm(x2, self.norm2, c.eps))
        if self.fused_glu:
            fmt = self._plain_fmt()
            need = binding.gemm_silu_mul_workspace_bytes(fmt, hc[0].shape[0], c.d_ff, c.d_model)
            act = binding.gemm_silu_mul(fmt, hc[0], hc[1], self.wgu[0], self.wgu[1],
                                        workspace=self._workspace(need, x.device) if need else None,
                                        prepared=self.prepared[id(self.wgu)] if self.prepared is not None else None)
        else:
            act = binding.silu_mul(self._gemm(hc, self.wgu))
        return binding.residual_add(x2, self._gemm(self._cast(act), self.wd))

    def matmul_flops(self, S, nominal=False):
        """2 * M * N * K summed over the seven quantized matmuls, counting what this layer EXECUTES: with the
        materialised map both attention products run in full (no causal skipping); the fused attention skips the key
        tiles of 32 that lie wholly behind the causal mask of a block of 32 queries, so a head multiplies
        S * (S + 32) / 2 query-key pairs instead of S * S. nominal=True counts the attention products in full
        whatever runs (the figure a dense-attention layer would be credited with)."""
        c = self.cfg
        W, F, kv = c.n_heads * c.head_dim, c.d_ff, c.n_kv_heads * c.head_dim
        lin = S * c.d_model * (W + 2 * kv) + S * W * c.d_model + S * c.d_model * 2 * F + S * F * c.d_model
        pairs = S * (S + 32) // 2 if (self.fused_attention and not nominal) else S * S
        att = 2 * c.n_heads * pairs * c.head_dim
        return 2.0 * (lin + att)


class LMHead:
    """What turns the last layer's output into log probabilities of tokens. weight: BF16 CUDA tensor [vocab, d_model], cast once here; norm: FP32
    [d_model], the normalisation in front of it; cap: logits x become cap tanh(x / cap). The logits exist for `rows_at_once` rows at a time. (Where
    the format multiplies in BF16 the weights are expanded for each such part: 4096 rows of 4096 against 128000 tokens 4.7 ms in parts of 1024, 3.7 at once.)"""

    def __init__(self, weight, norm, fmt, eps=1e-5, cap=0.0, rows_at_once=1024):
        self.fmt, self.eps, self.cap, self.rows_at_once = fmt, eps, cap, rows_at_once
        self.weight = binding.quantize(fmt, weight.contiguous())
        self.norm = norm.contiguous()

    def logits(self, x):
        """FP32 [rows, vocab] of x BF16 [rows, d_model], before the cap."""
        return binding.gemm(self.fmt, *binding.rmsnorm_quantize(self.fmt, x, self.norm, self.eps), *self.weight)

    def logprobs(self, x, targets=None, top=0):
        """binding.token_logprobs() of the rows x BF16 [rows, d_model]."""
        rows = x.shape[0]
        if targets is not None:  # (all of them: a part's would not show one too many)
            binding._ints(rows, targets)
        f = lambda *shape: torch.empty(shape, dtype=torch.float32, device=x.device)  # noqa: E731
        out = binding.TokenLogprobs(None if targets is None else f(rows), f(rows), f(rows, top) if top else None,
                                    torch.empty((rows, top), dtype=torch.int32, device=x.device) if top else None)
        for at in range(0, rows, self.rows_at_once):
            part = slice(at, at + self.rows_at_once)
            binding.token_logprobs(self.logits(x[part]), None if targets is None else targets[part], top, self.cap,
                                   out=tuple(None if t is None else t[part] for t in out))
        return out
