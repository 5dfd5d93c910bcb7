"""Serving with a cache held in 4 bits, on libsp (include/sp_serve.h): what a program that answers with
compressed layers runs beside them.

    cache = KvCache(pages, kv_heads, head_dim)         one per layer
    batch = Batch(cache, heads, requests, tokens, width)
    batch.plan(new, advance=True)                      tables of a step, on the GPU
    q = cache.append(q, k, v, batch.positions, batch.slots, cos_sin)     norms, rotation, 4-bit write
    o = cache.attend(q, batch, max_new)                attention over the cache
    logp, entropy, top, ids = token_logprobs(logits, tokens, 5)

Argument marshalling only: the work is in libsp's kernels, and PyTorch holds the buffers.  No call
synchronises, so a step can be captured in a CUDA graph.  Indices in device tensors (tables, slots,
positions, token ids) are checked by the kernels, which leave bad ones out; sp.check() then raises.
"""
from __future__ import annotations

import ctypes
import math

import torch

from . import sp
from .sp import SpAttendArgs, SpKv4, SpKvPlanArgs, SpRopeArgs, _check, _lib, _stream

PLAN_PAGES, PLAN_WIDTH, PLAN_TOKENS, PLAN_INPUT = 1, 2, 4, 8  # SP_PLAN_*


def _heads(x: torch.Tensor, heads: int | None, dim: int, name: str) -> int:
    """Checks x [tokens, heads, dim] bf16 with contiguous heads (a view of a fused row serves) and
    returns its token stride."""
    if x.dtype != torch.bfloat16 or x.dim() != 3 or x.shape[2] != dim or (heads is not None and x.shape[1] != heads):
        raise ValueError(f"{name}: bf16 [tokens, {'heads' if heads is None else heads}, {dim}] wanted, "
                         f"got {x.dtype} {list(x.shape)}")
    if x.stride(2) != 1 or (x.shape[1] > 1 and x.stride(1) != dim):
        raise ValueError(f"{name}: the heads of a token must be contiguous")
    return x.stride(0) if x.shape[0] > 1 else max(x.stride(0), x.shape[1] * dim)


def _index(x: torch.Tensor, n: int, dtype, name: str):
    if x.dtype != dtype or x.dim() != 1 or x.shape[0] < n or not x.is_contiguous():
        raise ValueError(f"{name}: contiguous {dtype} [{n}] wanted, got {x.dtype} {list(x.shape)}")


def _rope_args(q, k, v, positions, cos_sin, q_weight, k_weight, eps, pairs, q_out, k_out, cache, slots):
    t, dim = q.shape[0], q.shape[2]
    a = SpRopeArgs()
    a.q_stride, a.k_stride = _heads(q, None, dim, "q"), _heads(k, None, dim, "k")
    if k.shape[0] != t:
        raise ValueError("q and k hold different numbers of tokens")
    _index(positions, t, torch.int32, "positions")
    if cos_sin.dtype != torch.float32 or cos_sin.dim() != 2 or not cos_sin.is_contiguous():
        raise ValueError("cos_sin: contiguous float32 [rows, rot] wanted")
    for w, name in ((q_weight, "q_weight"), (k_weight, "k_weight")):
        if w is not None and (w.dtype != torch.bfloat16 or w.shape != (dim,) or not w.is_contiguous()):
            raise ValueError(f"{name}: contiguous bf16 [{dim}] wanted")
    if q_out is None:
        q_out = torch.empty((t, q.shape[1], dim), dtype=torch.bfloat16, device=q.device)
    elif q_out.dtype != torch.bfloat16 or q_out.shape != q.shape or not q_out.is_contiguous():
        raise ValueError("q_out: contiguous bf16 of q's shape wanted")
    a.q, a.k, a.q_out = q.data_ptr(), k.data_ptr(), q_out.data_ptr()
    a.positions, a.cos_sin, a.rows, a.rot = positions.data_ptr(), cos_sin.data_ptr(), cos_sin.shape[0], cos_sin.shape[1]
    a.q_weight = None if q_weight is None else q_weight.data_ptr()
    a.k_weight = None if k_weight is None else k_weight.data_ptr()
    a.eps, a.pairs = eps, 1 if pairs else 0
    a.tokens, a.heads, a.kv_heads, a.head_dim = t, q.shape[1], k.shape[1], dim
    if cache is None:
        if k_out is None:
            k_out = torch.empty((t, k.shape[1], dim), dtype=torch.bfloat16, device=k.device)
        elif k_out.dtype != torch.bfloat16 or k_out.shape != k.shape or not k_out.is_contiguous():
            raise ValueError("k_out: contiguous bf16 of k's shape wanted")
        a.k_out = k_out.data_ptr()
    else:
        a.v_stride = _heads(v, k.shape[1], dim, "v")
        if v.shape[0] != t:
            raise ValueError("k and v hold different numbers of tokens")
        _index(slots, t, torch.int64, "slots")
        a.v, a.slots, a.cache = v.data_ptr(), slots.data_ptr(), ctypes.pointer(cache._c)
    return a, q_out, k_out


def qk_norm_rope(q: torch.Tensor, k: torch.Tensor, positions: torch.Tensor, cos_sin: torch.Tensor,
                 q_weight: torch.Tensor | None = None, k_weight: torch.Tensor | None = None, eps: float = 1e-5,
                 pairs: bool = False, q_out: torch.Tensor | None = None, k_out: torch.Tensor | None = None, stream=None):
    """sp_qk_norm_rope: per-head norms (where a weight is given) and the rotation of q [T, H, D] and
    k [T, Hkv, D], bf16 views with contiguous heads, by rows `positions` (int32 [T]) of cos_sin
    (fp32 [rows, rot]: rot / 2 cosines, then as many sines).  pairs: channel 2i turns with 2i + 1
    instead of i with i + rot / 2.  Returns (q_out, k_out)."""
    a, q_out, k_out = _rope_args(q, k, None, positions, cos_sin, q_weight, k_weight, eps, pairs, q_out, k_out, None, None)
    _check(_lib.sp_qk_norm_rope(a, _stream(stream, q.device.index)), "sp_qk_norm_rope")
    return q_out, k_out


class KvCache:
    """Keys and values of one layer in 4 bits, in pages of `page_size` tokens (the format is in
    include/sp_serve.h).  `data`: a uint8 buffer to use instead of a new one."""

    def __init__(self, pages: int, kv_heads: int, head_dim: int, page_size: int = 64, device=None,
                 data: torch.Tensor | None = None):
        self._c = SpKv4(None, pages, page_size, kv_heads, head_dim, 0)
        b = ctypes.c_size_t()
        _check(_lib.sp_kv4_bytes(self._c, ctypes.byref(b)), "sp_kv4_bytes")
        if data is None:
            dev = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
            data = torch.empty(int(b.value), dtype=torch.uint8, device=dev)
        elif data.dtype != torch.uint8 or data.numel() != b.value or not data.is_contiguous():
            raise ValueError(f"data: {b.value} contiguous bytes wanted")
        self.pages, self.kv_heads, self.head_dim, self.page_size = pages, kv_heads, head_dim, page_size
        self.data = data
        self._c.data = data.data_ptr()
        self._ws_bytes = 0

    def append(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, positions: torch.Tensor, slots: torch.Tensor,
               cos_sin: torch.Tensor, q_weight: torch.Tensor | None = None, k_weight: torch.Tensor | None = None,
               eps: float = 1e-5, pairs: bool = False, out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
        """qk_norm_rope, with the keys and the values v (as they are) written to the cache at `slots`
        (int64 [T]; a negative one writes nothing).  Returns the queries."""
        a, out, _ = _rope_args(q, k, v, positions, cos_sin, q_weight, k_weight, eps, pairs, out, None, self, slots)
        _check(_lib.sp_qk_norm_rope(a, _stream(stream, q.device.index)), "sp_qk_norm_rope")
        return out

    def read(self, slots: torch.Tensor, stream=None) -> tuple[torch.Tensor, torch.Tensor]:
        """The cached keys and values at `slots` (int64 [n]) as bf16 [n, kv_heads, head_dim]."""
        _index(slots, 0, torch.int64, "slots")
        n = slots.shape[0]
        k, v = (torch.empty((n, self.kv_heads, self.head_dim), dtype=torch.bfloat16, device=slots.device)
                for _ in range(2))
        _check(_lib.sp_kv4_read(self._c, slots.data_ptr(), n, k.data_ptr(), v.data_ptr(),
                                _stream(stream, slots.device.index)), "sp_kv4_read")
        return k, v

    def attend(self, q: torch.Tensor, batch: "Batch", max_new: int, scale: float | None = None,
               out: torch.Tensor | None = None, workspace: torch.Tensor | None = None, stream=None) -> torch.Tensor:
        """Causal attention of q [T, H, D] (the step's tokens, request by request) over the cache by
        the tables of `batch`; max_new: at least the most new tokens of a request; scale: 1 / sqrt(D)
        by default.  A token that sees nothing gets zeros; rows behind the step's last token keep what
        `out` held."""
        a = batch._attend
        a.q_stride = _heads(q, batch.heads, self.head_dim, "q")
        if out is None:
            out = torch.empty(q.shape, dtype=torch.bfloat16, device=q.device)
        a.out_stride = _heads(out, batch.heads, self.head_dim, "out")
        if out.shape[0] != q.shape[0]:
            raise ValueError("q and out hold different numbers of tokens")
        if self.kv_heads != batch.kv_heads or self.page_size != batch.page_size:
            raise ValueError("the batch was planned for another kind of cache")
        a.q, a.out, a.tokens, a.max_new = q.data_ptr(), out.data_ptr(), q.shape[0], max_new
        a.cache = ctypes.pointer(self._c)
        a.table, a.lens = batch.table.data_ptr(), batch.lens.data_ptr()
        a.scale = 1.0 / math.sqrt(self.head_dim) if scale is None else scale
        if workspace is None:
            workspace = sp.workspace_for(self.workspace_size(), q.device, stream)
        _check(_lib.sp_kv4_attend(a, workspace.data_ptr(), workspace.numel(), _stream(stream, q.device.index)),
               "sp_kv4_attend")
        return out

    def workspace_size(self) -> int:
        if not self._ws_bytes:
            b = ctypes.c_size_t()
            _check(_lib.sp_kv4_attend_workspace_size(self.head_dim, ctypes.byref(b)), "sp_kv4_attend_workspace_size")
            self._ws_bytes = int(b.value)
        return self._ws_bytes


class Batch:
    """The tables of up to `requests` running requests over caches of one shape (the layers of a model
    share them): pages, lengths and, for a step of up to `tokens` new tokens, slots and positions.
    Everything is device data:

        cached [requests] int32       tokens before the step;  table [requests, width] int32, pages
        free [pages] int32, free_count [1]                      stack of unused pages
        lens, cu_q, slots, positions, next_count, status        what plan() writes

    A fresh batch has no tokens and every page on the stack."""

    def __init__(self, cache: KvCache, heads: int, requests: int, tokens: int, width: int):
        if heads < 1 or heads % cache.kv_heads:
            raise ValueError("heads: a multiple of the cache's key heads wanted")
        self.heads, self.kv_heads, self.page_size, self.pages = heads, cache.kv_heads, cache.page_size, cache.pages
        self.requests, self.tokens, self.width = requests, tokens, width
        dev = cache.data.device
        i32 = dict(dtype=torch.int32, device=dev)
        self.cached = torch.zeros(requests, **i32)
        self.table = torch.full((requests, width), -1, **i32)
        self.free = torch.arange(cache.pages - 1, -1, -1, **i32)
        self.free_count = torch.full((1,), cache.pages, **i32)
        self._lens = torch.zeros(requests, **i32)
        self._next_count = torch.zeros(1, **i32)
        self.lens, self.next_count = self._lens, self._next_count
        self.cu_q = torch.zeros(requests + 1, **i32)
        self.work = torch.zeros(2 * (requests + 1), **i32)
        self.slots = torch.full((tokens,), -1, dtype=torch.int64, device=dev)
        self.positions = torch.zeros(tokens, **i32)
        self.status = torch.zeros(1, **i32)
        a = self._plan = SpKvPlanArgs()
        a.cu_q, a.work, a.slots = self.cu_q.data_ptr(), self.work.data_ptr(), self.slots.data_ptr()
        a.positions, a.status = self.positions.data_ptr(), self.status.data_ptr()
        a.max_tokens, a.pages, a.requests, a.width = tokens, cache.pages, requests, width
        a.page_size, a.group = cache.page_size, heads // cache.kv_heads
        a = self._attend = SpAttendArgs()
        a.cu_q, a.work = self.cu_q.data_ptr(), self.work.data_ptr()
        a.requests, a.width, a.heads = requests, width, heads

    def plan(self, new: torch.Tensor, advance: bool = False, allocate: bool = True, stream=None) -> "Batch":
        """sp_kv_plan: the tables of a step that adds new[b] tokens (int32 [requests]) to request b, or
        ends it (new[b] < 0).  advance: the step's lengths and stack height replace the ones before it
        (cached, free_count); otherwise they stay, and the step can be planned again.  allocate=False:
        `table` already holds every page of the step.  A step that does not fit leaves everything as it
        is, has no tokens, and says why in `status` (PLAN_*)."""
        _index(new, self.requests, torch.int32, "new")
        a = self._plan
        self.lens = self.cached if advance else self._lens
        self.next_count = self.free_count if advance else self._next_count
        a.cached, a.new_tokens, a.table = self.cached.data_ptr(), new.data_ptr(), self.table.data_ptr()
        a.free_pages = self.free.data_ptr() if allocate else None
        a.free_count, a.next_count, a.lens = self.free_count.data_ptr(), self.next_count.data_ptr(), self.lens.data_ptr()
        _check(_lib.sp_kv_plan(a, _stream(stream, new.device.index)), "sp_kv_plan")
        return self


def token_logprobs(logits: torch.Tensor, tokens: torch.Tensor, top: int = 0, stream=None):
    """sp_token_logprobs: of each row of logits [T, V] (bf16 or float32, rows of unit stride), the log
    probability of tokens[t] (int64; a negative one asks for nothing and gets 0) and the entropy, both
    float32 [T]; with top > 0 also the `top` most likely entries: log probabilities [T, top] and ids
    (int64), by falling logit and, among equal ones, rising id."""
    if logits.dtype not in (torch.bfloat16, torch.float32) or logits.dim() != 2 or logits.stride(1) != 1:
        raise ValueError("logits: bf16 or float32 [T, V] with unit column stride wanted")
    t, v = logits.shape
    _index(tokens, t, torch.int64, "tokens")
    out = torch.empty((2, t), dtype=torch.float32, device=logits.device)
    logp, entropy = out[0], out[1]
    tl = ti = None
    if top:
        tl = torch.empty((t, top), dtype=torch.float32, device=logits.device)
        ti = torch.empty((t, top), dtype=torch.int64, device=logits.device)
    _check(_lib.sp_token_logprobs(logits.data_ptr(), 0 if logits.dtype == torch.bfloat16 else 1,
                                  logits.stride(0) if t > 1 else v, t, v, tokens.data_ptr(), top, logp.data_ptr(),
                                  entropy.data_ptr(), None if tl is None else tl.data_ptr(),
                                  None if ti is None else ti.data_ptr(), _stream(stream, logits.device.index)),
           "sp_token_logprobs")
    return (logp, entropy, tl, ti) if top else (logp, entropy)
