"""The timed cases of the serving operators: what a program that answers with a compressed model asks
of the package beside its linear layers, from the tables of its cache to the probabilities of its answer.

Operators (the "op" of a case):
  plan      block tables, slots and positions of a step, built on the GPU from the lengths of its
            requests: finished requests give their pages back, growing ones take pages
            (serve.Batch.plan).
  rope      per-head norms of queries and keys (where the model has them) and the position rotation in
            one pass: written as tensors (serve.qk_norm_rope), or the queries as a tensor and keys and
            values into the cache held in 4 bits (KvCache.append), whose rows are read back
            (KvCache.read).
  attend    causal attention of the newest tokens of each request over its cache held in 4 bits
            (KvCache.attend): single tokens, a few tokens, whole prompts.
  logprobs  log probabilities of given tokens, the entropy and the most likely alternatives
            (serve.token_logprobs).

32 heads of 128 and 4096 columns are the layer shapes that the benchmark and the tests use; 8 key heads
of 64 or 128, 32000 and 131071 vocabulary entries and the page sizes are generic.

The cache: one block per page and key head, [P][D/2] bytes of key codes, [P][D/2] of value codes, then
[P] keys' and [P] values' (scale, minimum) in fp16; byte j of a row holds value 2j in its low half and
2j + 1 in its high half; a code n stands for scale * n + minimum.
"""
import math
import random

import torch

own = False  # False: the operators' plain forms; True: the framework's kernels
EPS = 1e-5


def listed():
    """The cases, operator by operator."""
    return [
        # the tables of a decode step: 64 running requests grow by one token each
        {"name": "plan_decode_b64", "op": "plan", "requests": 64, "len_lo": 1, "len_hi": 8192, "new_hi": 1,
         "release": 0, "page": 64},
        # a busy scheduler's step: prompts are admitted, others grow, every ninth request has ended
        {"name": "plan_mixed_b1000", "op": "plan", "requests": 1000, "len_lo": 1, "len_hi": 4096, "new_hi": 256,
         "release": 9, "page": 16},
        # one decode token of one request, rotation only, from the fused q/k/v row of a layer
        {"name": "rope_decode_t1", "op": "rope", "to": "cache", "tokens": 1, "heads": 32, "kv_heads": 32, "dim": 128,
         "rot": 128, "norm": False, "pairs": False, "page": 64},
        # a step of a few hundred tokens of a model with shared key heads and norms per head
        {"name": "rope_norm_t513", "op": "rope", "to": "cache", "tokens": 513, "heads": 32, "kv_heads": 8, "dim": 128,
         "rot": 128, "norm": True, "pairs": False, "page": 16},
        # prefill of two 2048-token prompts
        {"name": "rope_prefill_t4096", "op": "rope", "to": "cache", "tokens": 4096, "heads": 32, "kv_heads": 32,
         "dim": 128, "rot": 128, "norm": False, "pairs": False, "page": 64},
        # single-stream decode at a middling context
        {"name": "attend_decode_b1", "op": "attend", "requests": 1, "len_lo": 4097, "len_hi": 4097, "new_hi": 1,
         "heads": 32, "kv_heads": 32, "dim": 128, "page": 64},
        # a decode step of a full server: 64 requests of very different lengths, shared key heads
        {"name": "attend_decode_b64", "op": "attend", "requests": 64, "len_lo": 100, "len_hi": 16384, "new_hi": 1,
         "heads": 32, "kv_heads": 8, "dim": 128, "page": 64},
        # several drafted tokens per request verified at once, heads of 64
        {"name": "attend_verify_b16", "op": "attend", "requests": 16, "len_lo": 500, "len_hi": 6000, "new_hi": 5,
         "heads": 32, "kv_heads": 8, "dim": 64, "page": 16},
        # prefill: two prompts of up to 2048 tokens, behind a cached prefix
        {"name": "attend_prefill_b2", "op": "attend", "requests": 2, "len_lo": 2048, "len_hi": 3001, "new_hi": 2048,
         "heads": 32, "kv_heads": 32, "dim": 128, "page": 64},
        # the answer of one decode step with its five best alternatives
        {"name": "logprobs_t1", "op": "logprobs", "tokens": 1, "vocab": 32000, "top": 5, "dtype": "bf16"},
        # a step of many requests over a large vocabulary of odd size, fp32 logits
        {"name": "logprobs_t64_fp32", "op": "logprobs", "tokens": 64, "vocab": 131071, "top": 20, "dtype": "fp32"},
        # scoring a text of 2048 tokens
        {"name": "logprobs_t2048", "op": "logprobs", "tokens": 2048, "vocab": 32000, "top": 0, "dtype": "bf16"},
    ]


def draw(rng):
    """One more case of the listed ranges."""
    op = rng.choice(["plan", "rope", "rope", "attend", "attend", "attend", "logprobs", "logprobs"])
    page = rng.choice([16, 32, 64, 128])
    if op == "plan":
        hi = _log_int(rng, 16, 8192)
        return {"op": op, "requests": _log_int(rng, 1, 1000), "len_lo": 1, "len_hi": hi,
                "new_hi": min(hi, _log_int(rng, 1, 256)), "release": rng.choice([0, 3, 9]), "page": page}
    dim = rng.choice([64, 128, 128])
    kv = rng.choice([1, 2, 8, 8, 32])
    heads = kv * rng.choice({1: [1, 7, 16], 2: [4, 8, 16], 8: [1, 2, 4], 32: [1]}[kv])
    if op == "rope":
        return {"op": op, "to": rng.choice(["cache", "cache", "tensor"]), "tokens": _log_int(rng, 1, 4096),
                "heads": heads, "kv_heads": kv, "dim": dim, "rot": rng.choice([dim, dim, dim // 2]),
                "norm": rng.random() < 0.5, "pairs": rng.random() < 0.3, "page": page}
    if op == "attend":
        new_hi = rng.choice([1, 1, _log_int(rng, 2, 8), _log_int(rng, 9, 2048)])
        hi = max(new_hi, _log_int(rng, 16, 16384 if new_hi <= 8 else 3000))
        most = (64 if kv <= 8 else 16) if new_hi <= 8 else 2 if new_hi > 500 else 8
        return {"op": op, "requests": _log_int(rng, 1, most), "len_lo": min(hi, _log_int(rng, 1, 2000)),
                "len_hi": hi, "new_hi": new_hi, "heads": heads, "kv_heads": kv, "dim": dim, "page": page}
    vocab = _log_int(rng, 1000, 131071)
    dtype = rng.choice(["bf16", "fp32"])
    most = max(1, min(2048, 65_536_000 // vocab // (1 if dtype == "bf16" else 2)))
    return {"op": op, "tokens": _log_int(rng, 1, most), "vocab": vocab, "top": rng.choice([0, 1, 5, 20]),
            "dtype": dtype}


def _log_int(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


# ------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(1000003 * (seed + 1))


def _lengths(case):
    """(tokens in the cache with this step's, this step's tokens) of each request, from the case alone:
    log-uniform lengths, the longest one among them; of five requests and more one is idle."""
    r = random.Random("%d %d %d %d" % (case["requests"], case["len_lo"], case["len_hi"], case["new_hi"]))
    lens, new = [], []
    for b in range(case["requests"]):
        n = case["len_hi"] if b == 0 else _log_int(r, case["len_lo"], case["len_hi"])
        a = case["new_hi"] if b == 0 or case["new_hi"] == 1 else r.randint(1, case["new_hi"])
        a = min(a, n)
        if case["op"] == "attend" and b == 4:
            a = 0
        lens.append(n)
        new.append(a)
    return lens, new


def _cos_sin(rows, rot):
    """[rows, rot] fp32: rot / 2 cosines, then as many sines, of a position's angles."""
    f = 10000.0 ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / rot)
    a = torch.arange(rows, device="cuda", dtype=torch.float64)[:, None] * f
    return torch.cat([a.cos(), a.sin()], 1).float()


def _quantize(x):
    """Codes, scale and minimum (fp32 values of fp16 numbers) of rows of fp32 values."""
    lo, hi = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    m = lo.clamp(-65504.0, 65504.0).half().float()
    s = ((hi - lo) * (1.0 / 15.0)).clamp(0.0, 65504.0).half().float()
    n = torch.where(s > 0, ((x - m) * (1.0 / s)).round().clamp(0.0, 15.0), torch.zeros_like(x))
    return n, s, m


def _plan_inputs(case, seed):
    lens, new = _lengths(case)
    cpu = torch.Generator().manual_seed(seed + 1)
    page, b = case["page"], case["requests"]
    width = -(-(case["len_hi"] + case["new_hi"]) // page)
    cached = torch.tensor([n - a for n, a in zip(lens, new)])
    new = torch.tensor(new)
    # which requests have ended and how far the others are differ from step to step
    cached += torch.randint(0, case["new_hi"] + 1, (b,), generator=cached_gen(seed))
    if case["release"]:
        new[torch.arange(b) % case["release"] == seed % case["release"]] = -1
    before = (cached + page - 1) // page
    total = b * width + 7
    order = torch.randperm(total, generator=cpu)
    held = int(before.sum())
    mask = torch.arange(width)[None, :] < before[:, None]
    table = torch.full((b, width), -1)
    table[mask] = order[:held]
    free = torch.zeros(total, dtype=torch.int64)
    free[:total - held] = order[held:]
    i32 = dict(dtype=torch.int32, device="cuda")
    return {"cached": cached.to(**i32), "new": new.to(**i32), "table": table.to(**i32), "free": free.to(**i32),
            "count": torch.tensor([total - held], **i32), "tokens": case["requests"] * case["new_hi"]}


def cached_gen(seed):
    return torch.Generator().manual_seed(7 * seed + 3)


def _rope_inputs(case, seed):
    g = _gen(seed)
    t, h, kv, d, page = case["tokens"], case["heads"], case["kv_heads"], case["dim"], case["page"]
    qkv = torch.randn((t, (h + 2 * kv), d), generator=g, device="cuda")
    # keys have channels of very different size, as trained models' have
    qkv[:, h:h + kv] *= torch.randn((kv, d), generator=g, device="cuda").mul_(0.5).exp_()
    out = {"qkv": qkv.to(torch.bfloat16).view(t, -1)}
    start = int(torch.randint(0, 4096, (1,), generator=g, device="cuda"))
    out["positions"] = torch.arange(start, start + t, device="cuda", dtype=torch.int32)
    out["cos_sin"] = _cos_sin(8192, case["rot"])
    out["qw"] = out["kw"] = None
    if case["norm"]:
        out["qw"], out["kw"] = (1 + 0.3 * torch.randn((2, d), generator=g, device="cuda")).to(torch.bfloat16)
    pages = -(-(t + page) // page)
    perm = torch.randperm(pages, generator=g, device="cuda")
    at = start % page + torch.arange(t, device="cuda")
    out["slots"] = perm[at // page] * page + at % page
    out["pages"] = pages
    return out


def _attend_codes(case, seed, pages):
    """Codes and parameters of a whole cache: (key codes, value codes [pages, kv, P, D] uint8, key and
    value parameters [pages, kv, P, 2] fp16)."""
    g = _gen(seed)
    kv, p, d = case["kv_heads"], case["page"], case["dim"]
    out = []
    for which in range(2):
        ns, ps = [], []
        ch = torch.randn((kv, 1, d), generator=g, device="cuda").mul_(0.4)
        for a in range(0, pages, 2048):
            x = torch.randn((min(2048, pages - a), kv, p, d), generator=g, device="cuda")
            x = x * ch.exp() if which == 0 else x + ch
            n, s, m = _quantize(x)
            ns.append(n.to(torch.uint8))
            ps.append(torch.cat([s, m], -1).half())
        out += [torch.cat(ns), torch.cat(ps)]
    return out


def _attend_inputs(case, seed, packed=True):
    lens, new = _lengths(case)
    g = _gen(seed + 500)
    page, b = case["page"], case["requests"]
    width = -(-max(lens) // page)
    need = [-(-n // page) for n in lens]
    pages = sum(need) + 3
    order = torch.randperm(pages, generator=g, device="cuda").int()
    table = torch.full((b, width), -1, dtype=torch.int32, device="cuda")
    at = 0
    kn, kp, vn, vp = _attend_codes(case, seed, pages)
    for i, n in enumerate(need):
        table[i, :n] = order[at:at + n]
        if lens[i] % page:  # what lies behind the last token was never written
            last = int(order[at + n - 1])
            for x in (kp, vp):
                x[last, :, lens[i] % page:] = float("nan")
        at += n
    t = sum(new)
    q = torch.randn((t, case["heads"], case["dim"]), generator=g, device="cuda").mul_(1.5).to(torch.bfloat16)
    i32 = dict(dtype=torch.int32, device="cuda")
    out = {"q": q, "table": table, "lens": torch.tensor(lens, **i32), "new": torch.tensor(new, **i32),
           "max_len": max(lens), "max_new": max(new), "pages": pages}
    if not packed:
        return out, (kn, kp, vn, vp), lens, new
    data = [(n[..., 0::2] | (n[..., 1::2] << 4)).reshape(pages, case["kv_heads"], -1) for n in (kn, vn)]
    data += [x.contiguous().view(torch.uint8).reshape(pages, case["kv_heads"], -1) for x in (kp, vp)]
    out["data"] = torch.cat(data, -1)
    return out


def _logits(case, seed):
    g = _gen(seed)
    t, v = case["tokens"], case["vocab"]
    x = torch.randn((t, v), generator=g, device="cuda").mul_(2.0)
    best = torch.randint(0, v, (t, 1), generator=g, device="cuda")
    x.scatter_add_(1, best, torch.full((t, 1), 6.0, device="cuda"))
    # of 16 rows one answers within a grammar: most of its vocabulary is shut
    shut = torch.rand((t, v), generator=g, device="cuda") < 0.9
    shut &= (torch.arange(t, device="cuda") % 16 == 5)[:, None]
    x.masked_fill_(shut, -math.inf)
    x = x.to(torch.bfloat16) if case["dtype"] == "bf16" else x
    tokens = torch.where(torch.arange(t, device="cuda") % 3 == 0, best[:, 0],
                         torch.randint(0, v, (t,), generator=g, device="cuda"))
    return {"logits": x, "tokens": tokens}


def prepare(case, seed):
    op = case["op"]
    if op == "plan":
        state = {**case, **_plan_inputs(case, seed)}
    elif op == "rope":
        state = {**case, **_rope_inputs(case, seed)}
    elif op == "attend":
        state = {**case, **_attend_inputs(case, seed)}
    else:
        state = {**case, **_logits(case, seed)}
    if own and op != "logprobs":  # the handles that a serving program keeps
        from paper_2405_03594_gb300 import serve

        if op == "plan":
            cache = serve.KvCache(state["free"].numel(), 1, 64, case["page"])
            b = serve.Batch(cache, 1, case["requests"], state["tokens"], state["table"].shape[1])
            b.table, b.cached, b.free, b.free_count = state["table"], state["cached"], state["free"], state["count"]
            state["batch"] = b
        else:
            state["cache"] = serve.KvCache(state["pages"], case["kv_heads"], case["dim"], case["page"],
                                           data=state.get("data"))
        if op == "attend":
            b = serve.Batch(state["cache"], case["heads"], case["requests"], state["q"].shape[0],
                            state["table"].shape[1])
            b.table.copy_(state["table"])
            b.cached.copy_(state["lens"] - state["new"])
            b.plan(state["new"], allocate=False)
            state["batch"] = b
    return state


def run(state):
    op = state["op"]
    if op == "plan":
        return _own_plan(state) if own else _plain_plan(state)
    if op == "rope":
        return _own_rope(state) if own else _plain_rope(state)
    if op == "attend":
        if own:
            return state["cache"].attend(state["q"], state["batch"], state["max_new"])
        return _plain_attend(state)
    if own:
        from paper_2405_03594_gb300 import serve

        return serve.token_logprobs(state["logits"], state["tokens"], state["top"])
    return _plain_logprobs(state)


# ------------------------------------------------------------------ the framework's kernels
def _own_plan(s):
    b = s["batch"]
    b.plan(s["new"])
    return b.lens, b.cu_q, b.slots, b.positions, b.table, b.free, b.next_count, b.status


def _own_rope(s):
    t, h, kv, d = s["tokens"], s["heads"], s["kv_heads"], s["dim"]
    x = s["qkv"].view(t, h + 2 * kv, d)
    q, k, v = x[:, :h], x[:, h:h + kv], x[:, h + kv:]
    kw = dict(q_weight=s["qw"], k_weight=s["kw"], eps=EPS, pairs=s["pairs"])
    if s["to"] == "cache":
        q = s["cache"].append(q, k, v, s["positions"], s["slots"], s["cos_sin"], **kw)
        return (q, *s["cache"].read(s["slots"]))
    from paper_2405_03594_gb300 import serve

    return serve.qk_norm_rope(q, k, s["positions"], s["cos_sin"], **kw)


# ------------------------------------------------------------------ plain forms
def _plain_plan(s):
    page, cached, new, table, total = s["page"], s["cached"].long(), s["new"].long(), s["table"], s["free"].numel()
    width = table.shape[1]
    gone, add = new < 0, new.clamp(min=0)
    lens = torch.where(gone, 0, cached + add)
    before, after = (cached + page - 1) // page, (lens + page - 1) // page
    back, take = torch.where(gone, before, 0), torch.where(gone, 0, after - before)
    j = torch.arange(width, device="cuda")[None, :]
    # the pages of finished requests go on the stack in their order
    pos = s["count"] + (back.cumsum(0) - back)[:, None] + j
    pos = torch.where(j < back[:, None], pos, total)
    free = torch.cat([s["free"], s["free"].new_zeros(1)])
    free = free.scatter(0, pos.flatten(), table.flatten())[:total]
    # and new ones come off its top
    top = s["count"].long() + back.sum()
    fresh = (j >= before[:, None]) & (j < after[:, None]) & ~gone[:, None]
    idx = top - 1 - ((take.cumsum(0) - take)[:, None] + j - before[:, None])
    grown = torch.where(fresh, free[torch.where(fresh, idx, 0)], table)
    cu = torch.cat([add.new_zeros(1), add.cumsum(0)])
    t = torch.arange(s["tokens"], device="cuda")
    b = torch.searchsorted(cu[1:], t, right=True).clamp(max=cached.numel() - 1)
    used = t < cu[-1]
    p = torch.where(used, cached[b] + t - cu[b], 0)
    slots = torch.where(used, grown[b, p // page].long() * page + p % page, -1)
    count = (top - take.sum()).int().view(1)
    return lens.int(), cu.int(), slots, p.int(), grown, free, count, torch.zeros_like(count)


def _plain_norm(x, w):
    # the sum of squares by halves, neighbours first
    y = x * x
    while y.shape[-1] > 1:
        y = y[..., 0::2] + y[..., 1::2]
    r = 1.0 / (y / x.shape[-1] + EPS).sqrt()
    return x * r * w.float()


def _plain_rotate(x, c, s, rot, pairs):
    r = x[..., :rot]
    a, b = (r[..., 0::2], r[..., 1::2]) if pairs else (r[..., :rot // 2], r[..., rot // 2:])
    u, v = a * c - b * s, b * c + a * s
    r = torch.stack([u, v], -1).flatten(-2) if pairs else torch.cat([u, v], -1)
    return torch.cat([r, x[..., rot:]], -1)


def _plain_rope(s):
    t, h, kv, d, rot = s["tokens"], s["heads"], s["kv_heads"], s["dim"], s["rot"]
    x = s["qkv"].view(t, h + 2 * kv, d).float()
    q, k, v = x[:, :h], x[:, h:h + kv], x[:, h + kv:]
    if s["qw"] is not None:
        q, k = _plain_norm(q, s["qw"]), _plain_norm(k, s["kw"])
    cs = s["cos_sin"][s["positions"].long()][:, None, :]
    c, sn = cs[..., :rot // 2], cs[..., rot // 2:]
    q, k = (_plain_rotate(y, c, sn, rot, s["pairs"]) for y in (q, k))
    if s["to"] == "tensor":
        return q.to(torch.bfloat16), k.to(torch.bfloat16)
    out = [q.to(torch.bfloat16)]
    for y in (k, v):
        n, sc, m = _quantize(y)
        out.append((sc * n + m).to(torch.bfloat16))
    return tuple(out)


def _plain_rows(s, first, size):
    """Rows [requests, keys, kv, D] of fp32 values from the packed cache, at the places the table names."""
    page, d, kv = s["page"], s["dim"], s["kv_heads"]
    at = torch.arange(s["max_len"], device="cuda")
    there = at[None, :] < s["lens"][:, None]
    pg = torch.where(there, s["table"].long()[:, at // page], 0)
    blocks = s["data"]
    code = blocks[:, :, first * page * d // 2:(first + 1) * page * d // 2].reshape(-1, kv, page, d // 2)
    par = blocks[:, :, page * d + first * page * 4:page * d + (first + 1) * page * 4].contiguous()
    par = par.view(torch.float16).reshape(-1, kv, page, 2)
    code = code[pg, :, (at % page)[None, :].expand_as(pg)]
    par = par[pg, :, (at % page)[None, :].expand_as(pg)].float()
    par = torch.where(there[:, :, None, None], par, 0.0)
    n = torch.stack([code & 15, code >> 4], -1).flatten(-2).float()
    return par[..., :1] * n + par[..., 1:]


def _plain_attend(s):
    h, kv, d, b, m = s["heads"], s["kv_heads"], s["dim"], s["requests"], s["max_new"]
    group = h // kv
    new, lens = s["new"].long(), s["lens"].long()
    k, v = _plain_rows(s, 0, d), _plain_rows(s, 1, d)
    cu = torch.cat([new.new_zeros(1), new.cumsum(0)])
    i = torch.arange(m, device="cuda")[None, :]
    has = i < new[:, None]
    at = torch.where(has, cu[:-1, None] + i, 0)
    q = s["q"].float()[at].view(b, m, kv, group, d).permute(0, 2, 3, 1, 4).reshape(b, kv, group * m, d)
    x = torch.matmul(q, k.permute(0, 2, 3, 1)) * (1.0 / math.sqrt(d))
    seen = (lens - new)[:, None] + i + 1
    shut = torch.arange(s["max_len"], device="cuda")[None, None, :] >= seen[:, :, None]
    x = x.view(b, kv, group, m, -1).masked_fill_(shut[:, None, None], -math.inf)
    x = x - x.amax(-1, keepdim=True)
    x = x.exp_()
    x = x / x.sum(-1, keepdim=True)
    o = torch.matmul(x.view(b, kv, group * m, -1), v.permute(0, 2, 1, 3))
    o = o.view(b, kv, group, m, d).permute(0, 3, 1, 2, 4).reshape(b, m, h, d)
    return o[has].to(torch.bfloat16)


def _plain_logprobs(s):
    x = s["logits"].float()
    m = x.amax(-1, keepdim=True)
    e = (x - m).exp()
    z = e.sum(-1, keepdim=True)
    logp = x - m - z.log()
    p = e / z
    entropy = -torch.where(p > 0, p * logp, 0.0).sum(-1)
    got = logp.gather(1, s["tokens"][:, None])[:, 0]
    if not s["top"]:
        return got, entropy
    at = torch.sort(x, dim=-1, descending=True, stable=True).indices[:, :s["top"]]
    return got, entropy, logp.gather(1, at), at


# ------------------------------------------------------------------ what is expected
def work(case):
    op = case["op"]
    if op == "plan":
        lens, new = _lengths(case)
        t = case["requests"] * case["new_hi"]
        pages = sum(-(-n // case["page"]) - -(-(n - a) // case["page"]) for n, a in zip(lens, new))
        return {"bytes": 16 * case["requests"] + 12 * t + 8 * pages, "flops": 0}
    if op == "rope":
        t, h, kv, d = case["tokens"], case["heads"], case["kv_heads"], case["dim"]
        b = 2 * t * d * (h + 2 * kv) + 4 * t * case["rot"] + 2 * t * h * d
        if case["to"] == "cache":  # the cache written, read, and its rows as bf16
            b += 2 * t * kv * (d + 8) + 4 * t * kv * d
        else:
            b += 2 * t * kv * d
            b -= 2 * t * kv * d  # no values
        return {"bytes": b, "flops": t * (h + kv) * (3 * case["rot"] + (4 * d if case["norm"] else 0))}
    if op == "attend":
        lens, new = _lengths(case)
        h, kv, d = case["heads"], case["kv_heads"], case["dim"]
        keys = sum(n for n, a in zip(lens, new) if a)
        seen = sum(a * (n - a) + a * (a + 1) // 2 for n, a in zip(lens, new))
        return {"bytes": keys * kv * (d + 8) + 4 * sum(new) * h * d, "flops": 4 * seen * h * d}
    es = 2 if case["dtype"] == "bf16" else 4
    t = case["tokens"]
    return {"bytes": t * case["vocab"] * es + t * (16 + 12 * case["top"]), "flops": 4 * t * case["vocab"]}


def exact(case, seed):
    """The same results from the definitions in 64 bits."""
    op = case["op"]
    if op == "plan":
        return None  # whole numbers
    if op == "rope":
        return _exact_rope(case, seed)
    if op == "attend":
        return _exact_attend(case, seed)
    t = _logits(case, seed)
    x = t["logits"].double()
    logp = torch.empty_like(x)
    for r in range(0, x.shape[0], 64):
        y = x[r:r + 64]
        logp[r:r + 64] = y - torch.logsumexp(y, -1, keepdim=True)
    entropy = -(logp.exp() * logp.masked_fill(logp == -math.inf, 0.0)).sum(-1)
    got = logp[torch.arange(x.shape[0], device="cuda"), t["tokens"]]
    if not case["top"]:
        return got, entropy
    return got, entropy, torch.topk(logp, case["top"], dim=-1).values, None


def _exact_rope(case, seed):
    s = _rope_inputs(case, seed)
    t, h, kv, d, rot = case["tokens"], case["heads"], case["kv_heads"], case["dim"], case["rot"]
    x = s["qkv"].double().view(t, h + 2 * kv, d)
    cs = s["cos_sin"].double()[s["positions"].long()]
    z = torch.complex(cs[:, :rot // 2], cs[:, rot // 2:])[:, None, :]
    out = []
    for y, w in ((x[:, :h], s["qw"]), (x[:, h:h + kv], s["kw"])):
        if w is not None:
            y = y / torch.sqrt(y.square().mean(-1, keepdim=True) + EPS) * w.double()
        y = y.clone()
        lo, hi = (slice(0, rot, 2), slice(1, rot, 2)) if case["pairs"] else (slice(0, rot // 2), slice(rot // 2, rot))
        turned = torch.complex(y[..., lo].contiguous(), y[..., hi].contiguous()) * z
        y[..., lo], y[..., hi] = turned.real, turned.imag
        out.append(y)
    if case["to"] == "tensor":
        return tuple(out)
    out.append(x[:, h + kv:])
    for i in (1, 2):
        y = out[i]
        lo, span = y.amin(-1, keepdim=True), y.amax(-1, keepdim=True) - y.amin(-1, keepdim=True)
        sc, m = (span / 15).half().double(), lo.half().double()
        out[i] = torch.where(sc > 0, torch.clamp(torch.round((y - m) / sc), 0, 15), 0.0) * sc + m
    return tuple(out)


def _exact_attend(case, seed):
    s, (kn, kp, vn, vp), lens, new = _attend_inputs(case, seed, packed=False)
    group, d, page = case["heads"] // case["kv_heads"], case["dim"], case["page"]
    outs, at = [], 0
    for b, (n, a) in enumerate(zip(lens, new)):
        if a == 0:
            continue
        pg = s["table"][b, :-(-n // page)].long()
        k, v = ((par[pg][..., :1].double() * code[pg].double() + par[pg][..., 1:].double())
                .permute(1, 0, 2, 3).flatten(1, 2)[:, :n] for code, par in ((kn, kp), (vn, vp)))
        q = s["q"][at:at + a].double() / math.sqrt(d)
        o = torch.empty((a, case["heads"], d), dtype=torch.float64, device="cuda")
        shut = torch.ones((a, n), dtype=torch.bool, device="cuda").triu(n - a + 1)
        for h in range(case["heads"]):
            x = (q[:, h] @ k[h // group].T).masked_fill_(shut, -math.inf)
            o[:, h] = torch.softmax(x, -1) @ v[h // group]
        outs.append(o)
        at += a
    return torch.cat(outs)
