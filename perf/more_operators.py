"""The timed cases of the operators for answering with drafted tokens: a small dense model drafts, the compressed
model looks at all drafted tokens in one step, and the tokens that its distribution stands by are kept.

Operators (the "op" of a case):
  fp8      y = x . W^T of layers that pruning leaves dense (the draft model's, the vocabulary's), in 8-bit
           floating point (e4m3): W with a scale for each 128 x 128 block, x quantised on the way with a
           scale for each 128 columns of a row (fp8.Fp8Matrix.linear).
  probs    probabilities from logits, with a temperature for each row and entries far below the best one
           left out (serve.token_probs).
  verify   of each request's drafted tokens the longest accepted run, and the token behind it, from the
           probabilities of both models and given random numbers (serve.verify_drafts); without drafts:
           sampling.
  retract  the pages and lengths of tokens that were not accepted, given back (serve.Batch.retract).

4096 columns, 12288, 22016 and 32000 rows are the layer shapes that the benchmark and the tests use; the others are
generic.

Quantisation, in fp32 with each operation rounded on its own, of the largest magnitude a of a block:
  s = max(a * (1 / 448), 2^-100)   code = e4m3(x * (1 / s))      value = s * code
Weights of a row for sampling: floor(2^40 * w) with w limited to [0, 1], so that their sums are whole numbers.
"""
import math
import random

import torch

own = False  # False: the operators' plain forms; True: the framework's kernels


def listed():
    """The cases, operator by operator."""
    return [
        # one decode token through a square layer of the draft model: latency
        {"name": "fp8_m1", "op": "fp8", "m": 1, "n": 4096, "k": 4096},
        # 16 requests' vocabulary: the weight's bytes
        {"name": "fp8_head_m16", "op": "fp8", "m": 16, "n": 32000, "k": 4096},
        # a verification step of 64 requests with up to five tokens each, sizes of no round number
        {"name": "fp8_ragged_m299", "op": "fp8", "m": 299, "n": 5003, "k": 1999},
        # a chunk of a prompt through the fused q/k/v layer
        {"name": "fp8_chunk_m512", "op": "fp8", "m": 512, "n": 12288, "k": 4096},
        # prompts through the fused gate/up layer
        {"name": "fp8_prefill_m4096", "op": "fp8", "m": 4096, "n": 22016, "k": 4096},
        # the rows of one request with four drafted tokens
        {"name": "probs_t5", "op": "probs", "tokens": 5, "vocab": 32000, "dtype": "bf16", "min_p": 0.0},
        # a step of 64 requests with four drafted tokens each, a large vocabulary of odd size
        {"name": "probs_t320_fp32", "op": "probs", "tokens": 320, "vocab": 131071, "dtype": "fp32", "min_p": 0.02},
        # one request
        {"name": "verify_b1", "op": "verify", "requests": 1, "drafts": 4, "vocab": 32000, "given": "fp32"},
        # a full server's step, the draft's probabilities kept in bf16
        {"name": "verify_b64", "op": "verify", "requests": 64, "drafts": 4, "vocab": 131071, "given": "bf16"},
        # sampling: a decode step of 256 requests without drafts
        {"name": "verify_sample_b256", "op": "verify", "requests": 256, "drafts": 0, "vocab": 32000, "given": "none"},
        # 64 requests give back what was not accepted
        {"name": "retract_b64", "op": "retract", "requests": 64, "len_hi": 8192, "drop_hi": 4, "page": 64},
        # many requests, long drafts over small pages
        {"name": "retract_b1000", "op": "retract", "requests": 1000, "len_hi": 4096, "drop_hi": 40, "page": 16},
    ]


def draw(rng):
    """One more case of the listed ranges."""
    op = rng.choice(["fp8", "fp8", "fp8", "fp8", "probs", "probs", "verify", "verify", "verify", "retract"])
    if op == "fp8":
        n, k = _log_int(rng, 64, 32000), _log_int(rng, 64, 11008)
        if rng.random() < 0.5:
            n, k = -(-n // 128) * 128, -(-k // 128) * 128
        k = min(k, 131072000 // n)
        m = min(_log_int(rng, 1, 4096), max(1, 4096 * 4096 * 22016 // (n * k)))
        return {"op": op, "m": m, "n": n, "k": k}
    if op == "retract":
        hi = _log_int(rng, 16, 8192)
        return {"op": op, "requests": _log_int(rng, 1, 1000), "len_hi": hi, "drop_hi": min(hi, _log_int(rng, 1, 40)),
                "page": rng.choice([16, 32, 64, 128])}
    vocab = _log_int(rng, 1000, 131071)
    if op == "probs":
        dtype = rng.choice(["bf16", "fp32"])
        most = max(1, 320 * 131071 // vocab // (1 if dtype == "fp32" else 2))
        return {"op": op, "tokens": min(most, _log_int(rng, 1, 2048)), "vocab": vocab, "dtype": dtype,
                "min_p": rng.choice([0.0, 0.0, 0.02, 0.2])}
    drafts = rng.choice([0, 1, 2, 4, 7])
    most = max(1, 64 * 131071 * 5 // (vocab * (drafts + 1)))
    given = rng.choice(["fp32", "bf16", "none"]) if drafts else "none"
    return {"op": op, "requests": min(most, _log_int(rng, 1, 256)), "drafts": drafts, "vocab": vocab, "given": given}


def _log_int(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


# ------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(1000003 * (seed + 1))


def _fp8_inputs(case, seed):
    g = _gen(seed)
    m, n, k = case["m"], case["n"], case["k"]
    # activations with columns of very different size, and a few large entries, as trained models' have
    x = torch.randn((m, k), generator=g, device="cuda") * torch.randn((k,), generator=g, device="cuda").mul_(0.7).exp_()
    x.mul_(torch.where(torch.rand((m, k), generator=g, device="cuda") < 1e-3, 20.0, 1.0))
    w = torch.randn((n, k), generator=g, device="cuda").mul_(0.02)
    w.mul_(torch.randn((n, 1), generator=g, device="cuda").mul_(0.3).exp_())
    a = _blocks(w, 128).abs().amax((1, 3))
    s = (a * (1.0 / 448.0)).clamp(min=2.0 ** -100)
    inv = (1.0 / s).repeat_interleave(128, 0)[:n].repeat_interleave(128, 1)[:, :k]
    return {"x": x.to(torch.bfloat16), "q": (w * inv).clamp(-448.0, 448.0).to(torch.float8_e4m3fn), "scale": s}


def _blocks(w, rows):
    """[ceil(n / rows), rows, ceil(k / 128), 128], zeros behind the ends."""
    n, k = w.shape
    out = w.new_zeros((-(-n // rows) * rows, -(-k // 128) * 128))
    out[:n, :k] = w
    return out.view(-1, rows, out.shape[1] // 128, 128)


def _logits(t, v, g):
    x = torch.randn((t, v), generator=g, device="cuda").mul_(1.5)
    best = torch.randint(0, v, (t, 4), generator=g, device="cuda")
    return x.scatter_(1, best, torch.tensor([[11.0, 10.5, 9.5, 9.0]], device="cuda").expand(t, 4))


def _probs_inputs(case, seed):
    g = _gen(seed)
    t, v = case["tokens"], case["vocab"]
    x = _logits(t, v, g)
    # of 16 rows one answers within a grammar: most of its vocabulary is shut
    shut = torch.rand((t, v), generator=g, device="cuda") < 0.9
    shut &= (torch.arange(t, device="cuda") % 16 == 5)[:, None]
    x.masked_fill_(shut, -math.inf)
    # every request has its temperature; one in eight wants the best token
    temperature = 0.5 + torch.rand(t, generator=g, device="cuda")
    temperature[torch.arange(t, device="cuda") % 8 == 3] = 0.0
    return {"logits": x.to(torch.bfloat16) if case["dtype"] == "bf16" else x, "temperature": temperature}


def _drafted(case):
    """(rows, drafts) of each request, from the case alone: of five requests and more one is idle and one
    has a chunk of its prompt before the drafted tokens."""
    r = random.Random("%d %d" % (case["requests"], case["drafts"]))
    new, drafts = [], []
    for b in range(case["requests"]):
        n = case["drafts"] if b == 0 else r.randint(0, case["drafts"])
        new.append(0 if b == 4 else n + 8 if b == 3 else n + 1)
        drafts.append(0 if b == 4 else n)
    return new, drafts


def _verify_inputs(case, seed):
    g = _gen(seed)
    new, drafts = _drafted(case)
    t, v = sum(new), case["vocab"]
    x = _logits(t, v, g)
    out = {"probs": torch.softmax(x, -1), "draft_probs": None}
    # the draft model's distribution is near the target's
    y = torch.softmax(x.add_(torch.randn((t, v), generator=g, device="cuda").mul_(0.5)), -1)
    out["ids"] = torch.multinomial(y, 1, generator=g)[:, 0].roll(1)
    if case["given"] != "none":
        out["draft_probs"] = y.to(torch.bfloat16) if case["given"] == "bf16" else y
    i32 = dict(dtype=torch.int32, device="cuda")
    out["cu_q"] = torch.tensor([0] + new, **i32).cumsum(0).int()
    out["drafted"] = torch.tensor(drafts, **i32)
    out["accept"] = torch.rand(t, generator=g, device="cuda")
    out["sample"] = torch.rand(case["requests"], generator=g, device="cuda")
    return out


def _retract_inputs(case, seed):
    cpu = torch.Generator().manual_seed(seed + 1)
    page, b = case["page"], case["requests"]
    width = -(-case["len_hi"] // page)
    cached = torch.randint(1, case["len_hi"] + 1, (b,), generator=cpu)
    drop = torch.minimum(torch.randint(0, case["drop_hi"] + 1, (b,), generator=cpu), cached)
    held = (cached + page - 1) // page
    total, used = b * width + 5, int(held.sum())
    order = torch.randperm(total, generator=cpu)
    table = torch.full((b, width), -1)
    mask = torch.arange(width)[None, :] < held[:, None]
    table[mask] = order[:used]
    free = torch.zeros(total, dtype=torch.int64)
    free[:total - used] = order[used:]
    i32 = dict(dtype=torch.int32, device="cuda")
    return {"cached": cached.to(**i32), "drop": drop.to(**i32), "table": table.to(**i32), "free": free.to(**i32),
            "count": torch.tensor([total - used], **i32)}


_INPUTS = {"fp8": _fp8_inputs, "probs": _probs_inputs, "verify": _verify_inputs, "retract": _retract_inputs}


def prepare(case, seed):
    state = {**case, **_INPUTS[case["op"]](case, seed)}
    if own and case["op"] == "fp8":  # the handles that a program keeps
        from paper_2405_03594_gb300 import fp8

        state["matrix"] = fp8.Fp8Matrix(state.pop("q"), state.pop("scale"))
    if own and case["op"] == "retract":
        from paper_2405_03594_gb300 import serve

        cache = serve.KvCache(state["free"].numel(), 1, 64, case["page"])
        b = serve.Batch(cache, 1, case["requests"], 1, state["table"].shape[1])
        b.table, b.cached, b.free, b.free_count = state["table"], state["cached"], state["free"], state["count"]
        state["batch"] = b
    return state


def run(state):
    op = state["op"]
    if op == "fp8":
        return _own_fp8(state) if own else _plain_fp8(state)
    if op == "retract":
        return _own_retract(state) if own else _plain_retract(state)
    if not own:
        return _plain_probs(state) if op == "probs" else _plain_verify(state)
    from paper_2405_03594_gb300 import serve

    if op == "probs":
        return serve.token_probs(state["logits"], state["temperature"], min_p=state["min_p"])
    return serve.verify_drafts(state["probs"], state["ids"], state["cu_q"], state["drafted"], state["accept"],
                               state["sample"], draft_probs=state["draft_probs"])


# ------------------------------------------------------------------ the framework's kernels
def _own_fp8(s):
    return s["matrix"].linear(s["x"])


def _own_retract(s):
    b = s["batch"]
    b.retract(s["drop"])
    return b.lens, b.free, b.next_count, b.status


# ------------------------------------------------------------------ plain forms
def _plain_fp8(s):
    n, k = s["n"], s["k"]
    x = _blocks(s["x"].float(), 1)[:, 0]
    sx = (x.abs().amax(-1, keepdim=True) * (1.0 / 448.0)).clamp(min=2.0 ** -100)
    x = (x * (1.0 / sx)).clamp(-448.0, 448.0).to(torch.float8_e4m3fn).float() * sx
    w = s["q"].float() * s["scale"].repeat_interleave(128, 0)[:n].repeat_interleave(128, 1)[:, :k]
    return torch.matmul(x.flatten(1)[:, :k], w.T).to(torch.bfloat16)


def _plain_probs(s):
    x = s["logits"].float()
    best = x.amax(-1, keepdim=True)
    z = (x - best) * (1.0 / s["temperature"].clamp(min=2.0 ** -120))[:, None]
    least = torch.tensor(math.log(s["min_p"]) if s["min_p"] else -math.inf, dtype=torch.float32, device="cuda")
    e = torch.where(z >= least, z.exp(), 0.0)
    p = e / e.sum(-1, keepdim=True)
    at = torch.arange(s["vocab"], device="cuda").expand_as(x)
    first = torch.where(x == best, at, s["vocab"]).amin(-1, keepdim=True)
    return torch.where((s["temperature"] > 0)[:, None], p, (at == first).float())


def _plain_verify(s):
    p, q, ids, n, v = s["probs"], s["draft_probs"], s["ids"], s["drafted"].long(), s["vocab"]
    cu = s["cu_q"].long()
    busy = cu[1:] > cu[:-1]
    first = torch.where(busy, cu[1:] - 1 - n, 0)
    i = torch.arange(max(s["drafts"], 1), device="cuda")[None, :]
    on = i < n[:, None]
    row = torch.where(on, first[:, None] + i, 0)
    d = ids[torch.where(on, row + 1, 0)]
    asked = 1.0 if q is None else q[row, d].float()
    ok = on & (s["accept"][row] * asked < p[row, d].float())
    accepted = torch.where(ok, 1, 0).cumprod(1).sum(1)
    row = first + accepted
    less = (accepted < n) & busy
    target = p[row].float()
    if q is None:
        at = torch.arange(v, device="cuda")[None, :]
        other = (at == ids[torch.where(less, row + 1, 0)][:, None]).float()
    else:
        other = q[row].float()
    rest = _whole(torch.where(less[:, None], target - other, target))
    rest = torch.where((rest.sum(-1) > 0)[:, None], rest, _whole(target))  # nothing left: the target's own
    up = rest.cumsum(-1)
    total = up[:, -1]
    u = (s["sample"].clamp(0.0, 1.0 - 2.0 ** -24) * 2.0 ** 24).long()
    t = (total >> 24) * u + (((total & (2 ** 24 - 1)) * u) >> 24)
    nxt = torch.where(busy & (total > 0), (up <= t[:, None]).sum(-1), -1)
    accepted = torch.where(busy, accepted, 0)
    return accepted.int(), torch.where(busy, n - accepted, 0).int(), nxt


def _whole(w):
    return (w.nan_to_num(0.0).clamp(0.0, 1.0) * 2.0 ** 40).long()


def _plain_retract(s):
    page, cached, table, total = s["page"], s["cached"].long(), s["table"], s["free"].numel()
    lens = cached - s["drop"].long()
    before, after = (cached + page - 1) // page, (lens + page - 1) // page
    back = before - after
    j = torch.arange(table.shape[1], device="cuda")[None, :]
    pos = s["count"] + (back.cumsum(0) - back)[:, None] + j - after[:, None]
    pos = torch.where((j >= after[:, None]) & (j < before[:, None]), pos, total)
    free = torch.cat([s["free"], s["free"].new_zeros(1)])
    free = free.scatter(0, pos.flatten(), table.flatten())[:total]
    count = (s["count"] + back.sum()).int()
    return lens.int(), free, count, torch.zeros_like(count)


# ------------------------------------------------------------------ what is expected
def work(case):
    op = case["op"]
    if op == "fp8":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": n * k + 4 * (-(-n // 128)) * (-(-k // 128)) + 2 * m * k + 2 * m * n, "flops": 2 * m * n * k}
    if op == "probs":
        es = 2 if case["dtype"] == "bf16" else 4
        return {"bytes": case["tokens"] * (case["vocab"] * (es + 4) + 4), "flops": 4 * case["tokens"] * case["vocab"]}
    if op == "verify":
        # a row of the target's probabilities per request; of the draft's too where a token was refused (which
        # tokens are depends on the random numbers: left out here)
        new, drafts = _drafted(case)
        busy = sum(1 for a in new if a)
        return {"bytes": busy * (4 * case["vocab"] + 32) + 24 * sum(drafts), "flops": busy * case["vocab"]}
    return {"bytes": 16 * case["requests"], "flops": 0}


def exact(case, seed):
    """The same results from the definitions in 64 bits."""
    op = case["op"]
    if op == "fp8":
        return _exact_fp8(case, seed)
    if op == "probs":
        return _exact_probs(case, seed)
    return None  # whole numbers


def _exact_fp8(case, seed):
    s = _fp8_inputs(case, seed)
    m, n, k = case["m"], case["n"], case["k"]
    y = torch.zeros((m, n), dtype=torch.float64, device="cuda")
    sw = s["scale"].double()
    for b in range(-(-k // 128)):
        x = s["x"][:, 128 * b:128 * (b + 1)].float()
        largest = torch.maximum(x.amax(1), -x.amin(1))
        sx = torch.maximum(largest * torch.tensor(1.0 / 448.0, device="cuda"), torch.tensor(2.0 ** -100, device="cuda"))
        v = (x * torch.reciprocal(sx)[:, None]).double()
        # to four significant bits, or to multiples of 2^-9
        step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
        code = torch.clamp(torch.round(v / step) * step, -448, 448)
        w = s["q"][:, 128 * b:128 * (b + 1)].double()
        y += (code @ w.T) * sx.double()[:, None] * sw[:, b].repeat_interleave(128)[:n]
    return y


def _exact_probs(case, seed):
    s = _probs_inputs(case, seed)
    out = torch.zeros((case["tokens"], case["vocab"]), dtype=torch.float64, device="cuda")
    for r in range(case["tokens"]):
        x, t = s["logits"][r].float(), float(s["temperature"][r])
        if t <= 0:
            out[r, int((x == x.max()).nonzero()[0])] = 1.0
            continue
        # which entries are kept is defined in fp32, what they are worth is not
        z = (x - x.max()) * torch.reciprocal(s["temperature"][r])
        y = x.double() / t
        if case["min_p"]:
            y[z < math.log(case["min_p"])] = -math.inf
        out[r] = torch.softmax(y, 0)
    return out
