"""Serving with a cache held in 4 bits, on libsp (include/sp_serve.h): what a program that answers with
compressed layers runs beside them.

    cache = KvCache(pages, kv_heads, head_dim)         one per layer
    batch = Batch(cache, heads, requests, tokens, width)
    batch.plan(new, advance=True)                      tables of a step, on the GPU
    q = cache.append(q, k, v, batch.positions, batch.slots, cos_sin)     norms, rotation, 4-bit write
    o = cache.attend(q, batch, max_new)                attention over the cache
    logp, entropy, top, ids = token_logprobs(logits, tokens, 5)
    p = token_probs(logits, temperature)               and with drafted tokens among the step's
    accepted, rejected, nxt = verify_drafts(p, ids, batch.cu_q, drafts, accept, sample, draft_probs)
    batch.retract(rejected, advance=True)

Argument marshalling only: the work is in libsp's kernels, and PyTorch holds the buffers.  No call
synchronises, so a step can be captured in a CUDA graph.  Every tensor of a call has to be on the current GPU.  Indices in device tensors (tables, slots,
positions, token ids) are checked by the kernels, which leave bad ones out; sp.check() then raises.
"""
from __future__ import annotations

import ctypes
import math
import struct

import torch

from . import sp
from .sp import SP_ERR_INVALID_ARG, SP_ERR_UNSUPPORTED, SpAttendArgs, SpKv4, SpKvPlanArgs, SpKvRetractArgs, SpRopeArgs, SpVerifyArgs, _check, _lib, _stream

PLAN_PAGES, PLAN_WIDTH, PLAN_TOKENS, PLAN_INPUT = 1, 2, 4, 8  # SP_PLAN_*
MOST_DRAWN = 1 << 22  # entries of a row that sp_verify_drafts draws from

_BF16, _F32, _I32, _I64 = torch.bfloat16, torch.float32, torch.int32, torch.int64
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
_CODES = {ctypes.c_void_p: "P", ctypes.c_int64: "q", ctypes.c_int32: "i", ctypes.c_float: "f"}


def _packed(name: str, args):
    """(packer of the argument struct's fields, the library function that takes the packed bytes).  A
    packed call costs a small part of a ctypes struct filled field by field: a decode step makes
    several calls per layer, each a few microseconds of GPU time."""
    fmt = struct.Struct("@" + "".join(_CODES.get(t, "P") for _, t in args._fields_) + "0q")  # (padded to whole words)
    assert fmt.size == ctypes.sizeof(args)
    fn = _lib[name]  # a function object of its own, with its own argument types
    fn.argtypes = [ctypes.c_char_p, *getattr(_lib, name).argtypes[1:]]
    fn.restype = ctypes.c_int
    return fmt.pack, fn


_pack_plan, _plan = _packed("sp_kv_plan", SpKvPlanArgs)
_pack_retract, _retract = _packed("sp_kv_retract", SpKvRetractArgs)
_pack_verify, _verify = _packed("sp_verify_drafts", SpVerifyArgs)
_pack_rope, _rope = _packed("sp_qk_norm_rope", SpRopeArgs)
_pack_attend, _attend = _packed("sp_kv4_attend", SpAttendArgs)
_read = _lib["sp_kv4_read"]  # (the cache by its address)
_read.argtypes, _read.restype = [ctypes.c_void_p, *_lib.sp_kv4_read.argtypes[1:]], ctypes.c_int


def _on_current(dev: int, x: torch.Tensor, name: str) -> int:
    """dev, where x is, which has to be the current GPU: a call's launches go there, and every other address
    that it hands over has to be that GPU's."""
    if dev < 0 or dev != _current_device():
        raise ValueError(f"{name} on {x.device}, the current GPU wanted")
    return dev


def _heads(x: torch.Tensor, heads: int | None, dim: int, dev: int, name: str) -> tuple[int, int, int]:
    """Checks x [tokens, heads, dim] bf16 on GPU `dev` with contiguous heads (a view of a fused row serves)
    and returns its tokens, heads and token stride."""
    shape, stride = x.shape, x.stride()
    if (x.dtype is not _BF16 or len(shape) != 3 or shape[2] != dim or (heads is not None and shape[1] != heads)
            or x.get_device() != dev):
        raise ValueError(f"{name}: bf16 [tokens, {'heads' if heads is None else heads}, {dim}] on GPU {dev} wanted, "
                         f"got {x.dtype} {list(shape)} on {x.device}")
    t, h, _ = shape
    if stride[2] != 1 or (h > 1 and stride[1] != dim):
        raise ValueError(f"{name}: the heads of a token must be contiguous")
    return t, h, stride[0] if t > 1 else max(stride[0], h * dim)


def _index(x: torch.Tensor, n: int, dtype, dev: int, name: str) -> int:
    """Checks a contiguous vector of n entries or more on GPU `dev` and returns its address."""
    if x.dtype is not dtype or x.dim() != 1 or x.shape[0] < n or not x.is_contiguous() or x.get_device() != dev:
        raise ValueError(f"{name}: contiguous {dtype} [{n}] on GPU {dev} wanted, got {x.dtype} {list(x.shape)} on {x.device}")
    return x.data_ptr()


def _weight(w: torch.Tensor | None, dim: int, dev: int, name: str) -> int:
    if w is None:
        return 0
    if w.dtype is not _BF16 or w.shape != (dim,) or not w.is_contiguous() or w.get_device() != dev:
        raise ValueError(f"{name}: contiguous bf16 [{dim}] on GPU {dev} wanted")
    return w.data_ptr()


def _output(out: torch.Tensor | None, t: int, h: int, dim: int, like: torch.Tensor, dev: int, name: str) -> torch.Tensor:
    if out is None:
        return torch.empty((t, h, dim), dtype=_BF16, device=like.device)  # (new_empty takes 1 us longer)
    if out.dtype is not _BF16 or out.shape != (t, h, dim) or not out.is_contiguous() or out.get_device() != dev:
        raise ValueError(f"{name}: contiguous bf16 {[t, h, dim]} on GPU {dev} wanted")
    return out


def _run_rope(q, k, v, positions, cos_sin, q_weight, k_weight, eps, pairs, q_out, k_out, cache, slots, stream):
    dim = q.shape[-1]
    dev = _on_current(q.get_device(), q, "q") if cache is None else _on_current(cache._gpu, cache._data, "the cache's buffer")
    t, h, q_stride = _heads(q, None, dim, dev, "q")
    tk, kv, k_stride = _heads(k, None, dim, dev, "k")
    if tk != t:
        raise ValueError("q and k hold different numbers of tokens")
    if cos_sin.dtype is not _F32 or cos_sin.dim() != 2 or not cos_sin.is_contiguous() or cos_sin.get_device() != dev:
        raise ValueError(f"cos_sin: contiguous float32 [rows, rot] on GPU {dev} wanted")
    rows, rot = cos_sin.shape
    pos = _index(positions, t, _I32, dev, "positions")
    qw, kw = _weight(q_weight, dim, dev, "q_weight"), _weight(k_weight, dim, dev, "k_weight")
    q_out = _output(q_out, t, h, dim, q, dev, "q_out")
    if cache is None:
        k_out = _output(k_out, t, kv, dim, k, dev, "k_out")
        v_ptr = v_stride = slot = where = 0
        k_ptr = k_out.data_ptr()
    else:
        tv, _, v_stride = _heads(v, kv, dim, dev, "v")
        if tv != t:
            raise ValueError("k and v hold different numbers of tokens")
        slot, where, v_ptr, k_ptr = _index(slots, t, _I64, dev, "slots"), cache._address, v.data_ptr(), 0
    _check(_rope(_pack_rope(q.data_ptr(), k.data_ptr(), v_ptr, q_stride, k_stride, v_stride, q_out.data_ptr(), k_ptr,
                            where, slot, pos, cos_sin.data_ptr(), rows, qw, kw, eps, t, h, kv, dim, rot,
                            1 if pairs else 0), _stream(stream, dev)), "sp_qk_norm_rope")
    return q_out, k_out


def qk_norm_rope(q: torch.Tensor, k: torch.Tensor, positions: torch.Tensor, cos_sin: torch.Tensor,
                 q_weight: torch.Tensor | None = None, k_weight: torch.Tensor | None = None, eps: float = 1e-5,
                 pairs: bool = False, q_out: torch.Tensor | None = None, k_out: torch.Tensor | None = None, stream=None):
    """sp_qk_norm_rope: per-head norms (where a weight is given) and the rotation of q [T, H, D] and
    k [T, Hkv, D], bf16 views with contiguous heads, by rows `positions` (int32 [T]) of cos_sin
    (fp32 [rows, rot]: rot / 2 cosines, then as many sines).  pairs: channel 2i turns with 2i + 1
    instead of i with i + rot / 2.  Returns (q_out, k_out)."""
    return _run_rope(q, k, None, positions, cos_sin, q_weight, k_weight, eps, pairs, q_out, k_out, None, None, stream)


class KvCache:
    """Keys and values of one layer in 4 bits, in pages of `page_size` tokens (the format is in
    include/sp_serve.h).  `data`: a uint8 buffer on the GPU of the calls to use instead of a new one."""

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
        self._data = data
        self._c.data = data.data_ptr()
        self._address = ctypes.addressof(self._c)
        self._gpu = data.get_device()
        self._ws_bytes = 0

    @property
    def data(self) -> torch.Tensor:
        """The buffer; its address is the cache's for life."""
        return self._data

    def append(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, positions: torch.Tensor, slots: torch.Tensor,
               cos_sin: torch.Tensor, q_weight: torch.Tensor | None = None, k_weight: torch.Tensor | None = None,
               eps: float = 1e-5, pairs: bool = False, out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
        """qk_norm_rope, with the keys and the values v (as they are) written to the cache at `slots`
        (int64 [T]; a negative one writes nothing).  Returns the queries."""
        return _run_rope(q, k, v, positions, cos_sin, q_weight, k_weight, eps, pairs, out, None, self, slots, stream)[0]

    def read(self, slots: torch.Tensor, stream=None) -> tuple[torch.Tensor, torch.Tensor]:
        """The cached keys and values at `slots` (int64 [n]) as bf16 [n, kv_heads, head_dim]."""
        dev = _on_current(self._gpu, self._data, "the cache's buffer")
        at = _index(slots, 0, _I64, dev, "slots")
        n = slots.shape[0]
        device = slots.device
        shape = (n, self.kv_heads, self.head_dim)
        k, v = torch.empty(shape, dtype=_BF16, device=device), torch.empty(shape, dtype=_BF16, device=device)
        _check(_read(self._address, at, n, k.data_ptr(), v.data_ptr(), _stream(stream, dev)), "sp_kv4_read")
        return k, v

    def attend(self, q: torch.Tensor, batch: "Batch", max_new: int, scale: float | None = None,
               out: torch.Tensor | None = None, workspace: torch.Tensor | None = None, stream=None) -> torch.Tensor:
        """Causal attention of q [T, H, D] (the step's tokens, request by request) over the cache by
        the tables of `batch`; max_new: at least the most new tokens of a request; scale: 1 / sqrt(D)
        by default.  Rows behind the step's last token keep what `out` held.  workspace: workspace_size()
        bytes (uint8) to use instead of the stream's own, zero at first as include/sp_serve.h says."""
        dim, dev = self.head_dim, _on_current(self._gpu, self._data, "the cache's buffer")
        t, h, q_stride = _heads(q, batch.heads, dim, dev, "q")
        if batch._gpu != dev:
            raise ValueError(f"the batch's tables are not on GPU {dev}")
        device = q.device
        if out is None:
            out, out_stride = torch.empty((t, h, dim), dtype=_BF16, device=device), h * dim
        else:
            to, _, out_stride = _heads(out, h, dim, dev, "out")
            if to != t:
                raise ValueError("q and out hold different numbers of tokens")
        if self.kv_heads != batch.kv_heads or self.page_size != batch.page_size:
            raise ValueError("the batch was planned for another kind of cache")
        if workspace is None:
            workspace = sp.workspace_for(self.workspace_size(), device, stream)
        elif workspace.dtype is not torch.uint8 or not workspace.is_contiguous() or workspace.get_device() != dev:
            raise ValueError(f"workspace: contiguous bytes (uint8) on GPU {dev} wanted")
        _check(_attend(_pack_attend(q.data_ptr(), out.data_ptr(), q_stride, out_stride, self._address,
                                    batch.table.data_ptr(), batch.lens.data_ptr(), batch.cu_q.data_ptr(),
                                    batch.work.data_ptr(), t, batch.requests, batch.width, h, max_new,
                                    1.0 / math.sqrt(dim) if scale is None else scale, 0),
                       workspace.data_ptr(), workspace.numel(), _stream(stream, dev)), "sp_kv4_attend")
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

    A fresh batch has no tokens and every page on the stack.  Another tensor of the same type on the
    same device, no smaller, may take the place of one of these; the sizes stay what they are."""

    _TABLES = {"cached": (_I32, lambda b: (b.requests,)), "table": (_I32, lambda b: (b.requests, b.width)),
               "free": (_I32, lambda b: (b.pages,)), "free_count": (_I32, lambda b: (1,)),
               "lens": (_I32, lambda b: (b.requests,)), "next_count": (_I32, lambda b: (1,)),
               "cu_q": (_I32, lambda b: (b.requests + 1,)), "work": (_I32, lambda b: (3 * (b.requests + 1),)),
               "slots": (_I64, lambda b: (b.tokens,)), "positions": (_I32, lambda b: (b.tokens,)),
               "status": (_I32, lambda b: (1,))}
    _SIZES = frozenset(("heads", "kv_heads", "page_size", "pages", "requests", "tokens", "width", "_gpu"))

    def __setattr__(self, name, value):
        # (the kernels go by the sizes: checked here once, so that no call has to)
        if name in self._TABLES:
            dtype, shape = self._TABLES[name][0], self._TABLES[name][1](self)
            if (not isinstance(value, torch.Tensor) or value.dtype is not dtype or value.dim() != len(shape)
                    or (value.shape[0] < shape[0] if len(shape) == 1 else tuple(value.shape) != shape)
                    or not value.is_contiguous() or value.get_device() != self._gpu):
                raise ValueError(f"{name}: contiguous {dtype} {list(shape)} on the batch's device wanted")
        elif name in self._SIZES and name in self.__dict__:
            raise AttributeError(f"{name}: a batch's sizes are those it was made with")
        object.__setattr__(self, name, value)

    def __init__(self, cache: KvCache, heads: int, requests: int, tokens: int, width: int):
        if heads < 1 or heads % cache.kv_heads:
            raise ValueError("heads: a multiple of the cache's key heads wanted")
        self.heads, self.kv_heads, self.page_size, self.pages = heads, cache.kv_heads, cache.page_size, cache.pages
        self.requests, self.tokens, self.width = requests, tokens, width
        dev = cache.data.device
        self._gpu = cache._gpu
        i32 = dict(dtype=torch.int32, device=dev)
        self.cached = torch.zeros(requests, **i32)
        self.table = torch.full((requests, width), -1, **i32)
        self.free = torch.arange(cache.pages - 1, -1, -1, **i32)
        self.free_count = torch.full((1,), cache.pages, **i32)
        self._lens = torch.zeros(requests, **i32)
        self._next_count = torch.zeros(1, **i32)
        self.lens, self.next_count = self._lens, self._next_count
        self.cu_q = torch.zeros(requests + 1, **i32)
        self.work = torch.zeros(3 * (requests + 1), **i32)
        self.slots = torch.full((tokens,), -1, dtype=torch.int64, device=dev)
        self.positions = torch.zeros(tokens, **i32)
        self.status = torch.zeros(1, **i32)

    def plan(self, new: torch.Tensor, advance: bool = False, allocate: bool = True, stream=None) -> "Batch":
        """sp_kv_plan: the tables of a step that adds new[b] tokens (int32 [requests]) to request b, or
        ends it (new[b] < 0).  advance: the step's lengths and stack height replace the ones before it
        (cached, free_count); otherwise they stay, and the step can be planned again.  allocate=False:
        `table` already holds every page of the step.  A step that does not fit leaves everything as it
        is, has no tokens, and says why in `status` (PLAN_*)."""
        dev = _on_current(self._gpu, self.cached, "the batch's tables")
        at = _index(new, self.requests, _I32, dev, "new")
        own = self.__dict__  # (these tensors have been checked)
        own["lens"] = self.cached if advance else self._lens
        own["next_count"] = self.free_count if advance else self._next_count
        _check(_plan(_pack_plan(self.cached.data_ptr(), at, self.table.data_ptr(),
                                self.free.data_ptr() if allocate else 0, self.free_count.data_ptr(),
                                self.next_count.data_ptr(), self.lens.data_ptr(), self.cu_q.data_ptr(),
                                self.work.data_ptr(), self.slots.data_ptr(), self.positions.data_ptr(),
                                self.status.data_ptr(), self.tokens, self.pages, self.requests, self.width,
                                self.page_size, self.heads // self.kv_heads),
                     _stream(stream, dev)), "sp_kv_plan")
        return self


    def retract(self, drop: torch.Tensor, advance: bool = False, allocate: bool = True, stream=None) -> "Batch":
        """sp_kv_retract: request b loses its last drop[b] tokens (int32 [requests], 0 to what it holds), such as
        drafts that were refused, and the pages that held nothing else go back on the stack.  advance and allocate
        as for plan(): the lengths and the stack's height after it are `lens` and `next_count`, or replace those
        before it.  Slots, positions and shares of a step planned before stay as they are; `status` gets PLAN_INPUT
        added where it cannot be done."""
        dev = _on_current(self._gpu, self.cached, "the batch's tables")
        at = _index(drop, self.requests, _I32, dev, "drop")
        own = self.__dict__
        own["lens"] = self.cached if advance else self._lens
        own["next_count"] = self.free_count if advance else self._next_count
        _check(_retract(_pack_retract(self.cached.data_ptr(), at, self.table.data_ptr(),
                                      self.free.data_ptr() if allocate else 0, self.free_count.data_ptr(),
                                      self.next_count.data_ptr(), self.lens.data_ptr(), self.status.data_ptr(),
                                      self.pages, self.requests, self.width, self.page_size, 0),
                        _stream(stream, dev)), "sp_kv_retract")
        return self


def token_logprobs(logits: torch.Tensor, tokens: torch.Tensor, top: int = 0, stream=None):
    """sp_token_logprobs: of each row of logits [T, V] (bf16 or float32, rows of unit stride), the log
    probability of tokens[t] (int64; a negative one asks for nothing and gets 0) and the entropy, both
    float32 [T]; with top > 0 also the `top` most likely entries: log probabilities [T, top] and ids
    (int64), by falling logit (-0 below +0, a NaN above all) and, among equal ones, rising id."""
    dtype = logits.dtype
    if (dtype is not _BF16 and dtype is not _F32) or logits.dim() != 2 or logits.stride(1) != 1:
        raise ValueError("logits: bf16 or float32 [T, V] with unit column stride on a GPU wanted")
    t, v = logits.shape
    dev = _on_current(logits.get_device(), logits, "logits")
    ids = _index(tokens, t, _I64, dev, "tokens")
    device = logits.device
    logp, entropy = torch.empty(t, dtype=_F32, device=device), torch.empty(t, dtype=_F32, device=device)
    tl = ti = None
    if top:
        tl, ti = torch.empty((t, top), dtype=_F32, device=device), torch.empty((t, top), dtype=_I64, device=device)
    _check(_lib.sp_token_logprobs(logits.data_ptr(), 0 if dtype is _BF16 else 1, logits.stride(0) if t > 1 else v, t, v,
                                  ids, top, logp.data_ptr(), entropy.data_ptr(), tl.data_ptr() if top else None,
                                  ti.data_ptr() if top else None, _stream(stream, dev)),
           "sp_token_logprobs")
    return (logp, entropy, tl, ti) if top else (logp, entropy)


def _row_type(x: torch.Tensor, dev: int, name: str) -> int:
    """Checks rows [T, V] of probabilities or logits and returns their type's number (SP_LOGITS_*)."""
    dtype = x.dtype
    if (dtype is not _BF16 and dtype is not _F32) or x.dim() != 2 or x.stride(1) != 1 or x.get_device() != dev:
        raise ValueError(f"{name}: bf16 or float32 [T, V] with unit column stride on GPU {dev} wanted")
    return 0 if dtype is _BF16 else 1


def _row_temperatures(temperature, t: int, dev: int) -> tuple[int, float]:
    """The address of a vector of t temperatures, or 0, and the number for all rows."""
    if not isinstance(temperature, torch.Tensor):
        return 0, float(temperature)
    if temperature.shape != (t,):  # (a longer one would be the requests', or another step's)
        raise ValueError(f"temperature: a number, or float32 [{t}], one for each row, wanted, got {list(temperature.shape)}")
    return _index(temperature, t, _F32, dev, "temperature"), 1.0


def token_probs(logits: torch.Tensor, temperature=1.0, min_p: float = 0.0, out: torch.Tensor | None = None,
                stream=None) -> torch.Tensor:
    """sp_token_probs: probabilities, float32 [T, V], of the rows of logits [T, V] (bf16 or float32, rows of unit
    stride).  temperature: a number, or one for each row (float32 [T], neither more nor fewer); 0 or less takes the best entry.
    min_p: entries of less than min_p times the best one's probability are left out.  out must not overlap logits or temperature.  The last
    bits of a row depend on how many rows the call has: those of a row alone and among others may differ."""
    dev = _on_current(logits.get_device(), logits, "logits")
    kind = _row_type(logits, dev, "logits")
    t, v = logits.shape
    if v < 1:
        raise ValueError("logits: a vocabulary of one entry or more wanted")
    per_row, one = _row_temperatures(temperature, t, dev)
    if out is None:
        out, out_stride = torch.empty((t, v), dtype=_F32, device=logits.device), v
    elif _row_type(out, dev, "out") != 1 or out.shape != logits.shape:
        raise ValueError(f"out: float32 {[t, v]} wanted")
    else:
        out_stride = out.stride(0) if t > 1 else max(out.stride(0), v)
    _check(_lib.sp_token_probs(logits.data_ptr(), kind, logits.stride(0) if t > 1 else v, t, v, per_row, one, min_p,
                               out.data_ptr(), out_stride, _stream(stream, dev)),
           "sp_token_probs")
    return out


def _draft_rows(draft_probs: torch.Tensor | None, t: int, v: int, dev: int) -> tuple[int, int, int]:
    """Address, row stride and type of the drafts' probabilities [t, v]; zeros where drafts are certain."""
    if draft_probs is None:
        return 0, 0, 0
    kind = _row_type(draft_probs, dev, "draft_probs")
    if draft_probs.shape != (t, v):
        raise ValueError(f"draft_probs: {[t, v]} wanted")
    return draft_probs.data_ptr(), draft_probs.stride(0) if t > 1 else v, kind


def check_drawing(t: int, v: int, requests: int, dev: int, sample: torch.Tensor, temperature, min_p: float,
                  drafts: torch.Tensor | None = None, accept: torch.Tensor | None = None, draft_probs: torch.Tensor | None = None):
    """Refuses the arguments that token_probs and verify_drafts would refuse for a step of t rows over v entries: what
    changes tables before it has its logits asks first."""
    _, one = _row_temperatures(temperature, t, dev)
    if one != one or not 0 <= min_p <= 1:
        _check(SP_ERR_INVALID_ARG, "sp_token_probs")
    _index(sample, requests, _F32, dev, "sample")
    if drafts is not None or accept is not None:
        _index(drafts, requests, _I32, dev, "drafts")
        _index(accept, t, _F32, dev, "accept")
        draft, stride, _ = _draft_rows(draft_probs, t, v, dev)
        if draft and stride < v:
            _check(SP_ERR_INVALID_ARG, "sp_verify_drafts")
    if v > MOST_DRAWN:
        _check(SP_ERR_UNSUPPORTED, "sp_verify_drafts")


def verify_drafts(probs: torch.Tensor, ids: torch.Tensor, cu_q: torch.Tensor, drafts: torch.Tensor, accept: torch.Tensor,
                  sample: torch.Tensor, draft_probs: torch.Tensor | None = None, stream=None):
    """sp_verify_drafts: of each request's drafted tokens, the last drafts[b] (int32 [B]) of its step's tokens
    ids[cu_q[b]:cu_q[b + 1]] (int64 [T]; int32 [B + 1]), which ones the target's probabilities (bf16 or float32 [T, V],
    row j behind token j) keep, and the token behind those.  accept (float32 [T]): accept[j] decides on token j + 1;
    sample (float32 [B]) draws the token behind; both uniform in [0, 1).  draft_probs [T, V]: row j is what token j + 1
    was drawn from; None: drafts are certain.  With drafts of 0 it samples.  Returns
    (accepted int32 [B], rejected int32 [B], next token int64 [B], -1 for a request without tokens)."""
    dev = _on_current(probs.get_device(), probs, "probs")
    kind = _row_type(probs, dev, "probs")
    t, v = probs.shape
    b = cu_q.shape[0] - 1 if cu_q.dim() == 1 else -1
    if b < 0:
        raise ValueError("cu_q: int32 [requests + 1] wanted")
    draft, draft_stride, draft_kind = _draft_rows(draft_probs, t, v, dev)
    where = (_index(ids, t, _I64, dev, "ids"), _index(cu_q, b + 1, _I32, dev, "cu_q"), _index(drafts, b, _I32, dev, "drafts"),
             _index(accept, t, _F32, dev, "accept"), _index(sample, b, _F32, dev, "sample"))
    device = probs.device
    accepted, rejected = torch.empty(b, dtype=_I32, device=device), torch.empty(b, dtype=_I32, device=device)
    nxt = torch.empty(b, dtype=_I64, device=device)
    _check(_verify(_pack_verify(probs.data_ptr(), draft, probs.stride(0) if t > 1 else v, draft_stride, t, v, *where,
                                accepted.data_ptr(), rejected.data_ptr(), nxt.data_ptr(), b, kind, draft_kind, 0),
                   _stream(stream, dev)), "sp_verify_drafts")
    return accepted, rejected, nxt
