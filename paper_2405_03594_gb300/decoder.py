"""Prefill and decode with compressed layers and a cache held in 4 bits: the layers of the linear stack
(stack.py) with the serving operators (serve.py) where that stack leaves attention out.

    h    = embed[ids]
    per layer
        q, k, v = h.Wqkv^T                             (sparse linear)
        q       = rotation(q); k, v to the cache        (KvCache.append)
        o       = attention over the cache              (KvCache.attend)
        h       = h + o.Wo^T                            (sparse linear, residual)
        a       = gate(h) * up(h)                       (sparse linear, interleaved gate/up rows)
        h       = h + a.Wdown^T                         (sparse linear, residual)
    logits = h.Whead^T                                  (sparse linear)

Every linear may be a dense one in 8 bits instead (fp8.Fp8Matrix), as pruning leaves the vocabulary's, and as a small
model that drafts tokens has them.

A step takes any mixture of prompts, chunks of prompts and single tokens of its requests; prompts and
decode steps are the same call.  As in the linear stack there is no normalisation between the
layers; per-head norms of queries and keys are the caller's choice.  All arithmetic runs in
libsp kernels but the embedding's rows, which PyTorch gathers."""
from __future__ import annotations

import torch

from . import sp
from .fp8 import Fp8Matrix
from .serve import Batch, KvCache, check_drawing, token_logprobs, token_probs, verify_drafts

NAMES = ("qkv", "o", "gate_up", "down")


def rotation_table(rows: int, rot: int, base: float = 10000.0, device="cuda") -> torch.Tensor:
    """cos_sin [rows, rot] float32 of serve.qk_norm_rope: angle i of position p is p * base^(-2i / rot)."""
    f = base ** (-torch.arange(0, rot, 2, device=device, dtype=torch.float64) / rot)
    a = torch.arange(rows, device=device, dtype=torch.float64)[:, None] * f
    return torch.cat([a.cos(), a.sin()], 1).float()


class Decoder:
    """layers: one dict of matrices per layer, SparseMatrix or (dense, in 8 bits) Fp8Matrix, with the names of NAMES -- qkv [(H + 2 Hkv) D, d], o [d, H D],
    gate_up [2F, d] (rows interleaved: gate_j, up_j), down [d, F]; embed [V, d] bf16; head: a matrix of either kind [V, d].
    Up to `requests` requests of up to `width` pages each share `pages` pages; a step has up to `tokens` new
    tokens.  The rotation's table has `positions` rows, or as many as the `width` pages of a request hold if
    that is more, so that every token has its own."""

    def __init__(self, layers, embed: torch.Tensor, head: sp.SparseMatrix | Fp8Matrix, heads: int, kv_heads: int, pages: int,
                 requests: int, tokens: int, width: int, page_size: int = 64, positions: int = 8192,
                 q_weight: torch.Tensor | None = None, k_weight: torch.Tensor | None = None):
        self.layers, self.embed, self.head = layers, embed, head
        self.heads, self.kv_heads = heads, kv_heads
        self.d = embed.shape[1]
        n_qkv = layers[0]["qkv"].n
        self.dim = n_qkv // (heads + 2 * kv_heads)
        if any(m["qkv"].n != n_qkv or m["o"].k != heads * self.dim or m["o"].n != self.d or
               m["gate_up"].n != 2 * m["down"].k for m in layers):
            raise ValueError("layers: shapes that do not belong together")
        dev = embed.device
        self.norms = dict(q_weight=q_weight, k_weight=k_weight)
        self.cos_sin = rotation_table(max(positions, width * page_size), self.dim, device=dev)
        self.caches = [KvCache(pages, kv_heads, self.dim, page_size, device=dev) for _ in layers]
        self.batch = Batch(self.caches[0], heads, requests, tokens, width)
        bf = dict(dtype=torch.bfloat16, device=dev)
        self.h = torch.empty((tokens, self.d), **bf)
        self.qkv = torch.empty((tokens, n_qkv), **bf)
        self.gu = torch.empty((tokens, layers[0]["gate_up"].n), **bf)
        self.a = torch.empty((tokens, layers[0]["down"].k), **bf)
        self.t = torch.empty((tokens, self.d), **bf)
        self.q = torch.empty((tokens, heads, self.dim), **bf)
        self.o = torch.empty((tokens, heads, self.dim), **bf)
        self.logits = torch.empty((tokens, head.n), **bf)
        self.zero = torch.zeros(self.d, **bf)  # the linear stack's residual vectors are not part of a model

    def step(self, ids: torch.Tensor, new: torch.Tensor, max_new: int, record=None) -> torch.Tensor:
        """Runs the step's tokens ids (int64 [t], request by request) of requests that each get new[b] of them
        (int32 [requests]; < 0: the request has ended and gives its pages back); max_new: at least the most
        of one request.  Returns the logits [t, V].  Ids that the step cannot take are refused before anything changes.  A step that does not fit (batch.status) writes no cache.
        If `record` is a list, (h before the layer, queries, attention's output) of each layer and h before the
        head are appended to it (copies)."""
        if ids.dim() != 1 or ids.shape[0] > self.h.shape[0] or ids.dtype not in (torch.int64, torch.int32) or ids.device != self.h.device:
            raise ValueError(f"ids: up to {self.h.shape[0]} int64 on {self.h.device} wanted, got {ids.dtype} {list(ids.shape)} on {ids.device}")
        t = ids.shape[0]
        b, h, qkv, gu, a, tmp, q, o = (self.batch, *(x[:t] for x in (self.h, self.qkv, self.gu, self.a, self.t, self.q, self.o)))
        b.plan(new, advance=True)
        if t == 0:  # requests that end or wait
            return self.logits[:0]
        torch.index_select(self.embed, 0, ids, out=h)
        H, G, D = self.heads, self.kv_heads, self.dim
        x = qkv.view(t, H + 2 * G, D)
        for m, cache in zip(self.layers, self.caches):
            before = h.clone() if record is not None else None
            m["qkv"].linear(h, out=qkv)
            cache.append(x[:, :H], x[:, H:H + G], x[:, H + G:], b.positions, b.slots, self.cos_sin, out=q, **self.norms)
            cache.attend(q, b, max_new, out=o)
            if record is not None:
                record.append((before, q.clone(), o.clone()))
            m["o"].linear(o.view(t, H * D), out=tmp)
            sp.residual_add(h, tmp, self.zero)
            m["gate_up"].linear(h, out=gu)
            sp.mul_pairs(a, gu)
            m["down"].linear(a, out=tmp)
            sp.residual_add(h, tmp, self.zero)
        if record is not None:
            record.append(h.clone())
        return self.head.linear(h, out=self.logits[:t])

    def sample(self, ids: torch.Tensor, new: torch.Tensor, max_new: int, sample: torch.Tensor, temperature=1.0, min_p: float = 0.0):
        """step(), then a token for each request behind its last one, drawn by `sample` (float32 [requests] in [0, 1)) from
        the probabilities at that temperature (token_probs): (next ids [requests], -1 for a request without new tokens;
        probabilities [t, V], float32).  temperature: a number, or one for each of the step's tokens (float32 [t], as the ids
        lie); of one for each request, float32 [requests], those are
        torch.repeat_interleave(temperature, new.clamp(min=0), output_size=t).  Arguments that cannot be are refused
        before anything changes, as step() refuses ids."""
        t, b = ids.numel(), self.batch
        check_drawing(t, self.head.n, b.requests, b._gpu, sample, temperature, min_p)
        probs = token_probs(self.step(ids, new, max_new), temperature, min_p)
        none = torch.zeros(b.requests, dtype=torch.int32, device=self.h.device)
        nxt = verify_drafts(probs, ids.long().contiguous(), b.cu_q[:b.requests + 1], none,
                            torch.empty(t, dtype=torch.float32, device=self.h.device), sample)[2]
        return nxt, probs

    def verify(self, ids: torch.Tensor, new: torch.Tensor, max_new: int, drafts: torch.Tensor, accept: torch.Tensor,
               sample: torch.Tensor, draft_probs: torch.Tensor | None = None, temperature=1.0, min_p: float = 0.0):
        """step(), where the last drafts[b] (int32 [requests]) of a request's new tokens are drafted ones: keeps the run of them
        that the model's probabilities accept (verify_drafts: accept float32 [t], sample float32 [requests], draft_probs [t, V]
        with row j what token j + 1 was drawn from), takes the others back out of the cache's tables, and draws the token
        behind.  A request's first new token is the one drawn before.  temperature: as for sample().  Returns (accepted, rejected
        int32 [requests], next ids [requests])."""
        b = self.batch
        check_drawing(ids.numel(), self.head.n, b.requests, b._gpu, sample, temperature, min_p, drafts, accept, draft_probs)
        probs = token_probs(self.step(ids, new, max_new), temperature, min_p)
        accepted, rejected, nxt = verify_drafts(probs, ids.long().contiguous(), b.cu_q[:b.requests + 1], drafts, accept, sample, draft_probs)
        b.retract(rejected, advance=True)
        return accepted, rejected, nxt

    def greedy(self, ids: torch.Tensor, new: torch.Tensor, max_new: int, top: int = 1):
        """step(), then of each of its tokens the likeliest next one with its log probability, the entropy, and
        the `top` likeliest: (next ids [t], log probabilities [t], entropy [t], top log probabilities, top ids)."""
        logits = self.step(ids, new, max_new)
        # (a token id of -1 asks for no log probability: the likeliest one's is the first of the top)
        none = torch.full((ids.shape[0],), -1, dtype=torch.int64, device=ids.device)
        _, entropy, tl, ti = token_logprobs(logits, none, max(top, 1))
        return ti[:, 0], tl[:, 0], entropy, tl, ti
