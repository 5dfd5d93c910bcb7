"""Probabilities, verification of drafted tokens and tokens taken back, on the GPU against the models of
tests/drafts_ref.py.

Verification and tables are whole numbers and compared for equality.  A probability exp(z) / S has z from two fp32
roundings, |z| 2^-23 off (relative, in the exponential), the product with log2(e) as much again, ex2 2^-22, the sum over
up to a few hundred terms a thread and the division some 2^-20 together: (3 |z| 2^-24 + 2^-19) p, where p is a
normal number; where it is smaller ex2 may give 0, so 2^-125 more."""
import numpy as np
import pytest
import torch

from tests import drafts_ref as ref
from tests import gpu_util as gu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sp():
    from paper_2405_03594_gb300 import sp as _sp

    return _sp


@pytest.fixture(scope="module")
def serve():
    from paper_2405_03594_gb300 import serve as _s

    return _s


def _dev(a, dtype):
    return torch.tensor(np.asarray(a), dtype=dtype, device="cuda")


def _i32(a):
    return _dev(a, torch.int32)


def _i64(a):
    return _dev(a, torch.int64)


# ------------------------------------------------------------------ probabilities
def _check_probs(got, x, temperature, min_p):
    want = ref.probs(x, temperature, min_p)
    got = got.double().cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(want))
    with np.errstate(all="ignore"):
        t = np.maximum(np.where(np.asarray(temperature) > 0, temperature, 1), 2.0 ** -120)[:, None]
        z = np.nan_to_num(np.abs(x - x.max(-1, keepdims=True)) / t, nan=0, posinf=0)
        z = np.minimum(z, 120)
    f = ~np.isnan(want)
    assert (np.abs(got - want)[f] <= ((3 * z * 2.0 ** -24 + 2.0 ** -19) * want + 2.0 ** -125)[f]).all()
    kept = np.where(f, want, 0) > 2.0 ** -120
    assert (got[kept] > 0).all() and not got[f & (want == 0) & ~kept].any()


@pytest.mark.parametrize("t,v", [(1, 1), (1, 2), (3, 7), (2, 63), (1, 1000), (5, 4099), (130, 515), (1, 32000), (4, 32003), (700, 130),
                                 (2, 131071), (1, 300001)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("min_p", [0.0, 0.03, 1.0])
def test_probs(sp, serve, t, v, dtype, min_p):
    g = np.random.default_rng(t + v)
    x = (3 * g.standard_normal((t, v))).astype(np.float32)
    x[:, g.integers(v)] += 6
    x[t // 2, g.random(v) < 0.5] = -np.inf
    x[t // 2, 0] = 1.0
    if v > 5:
        x[0, 5] = x[0].max()  # two best ones
    xt = _dev(x, torch.bfloat16 if dtype == "bf16" else torch.float32)
    temperature = np.where(np.arange(t) % 3 == 1, 0.0, 0.3 + g.random(t)).astype(np.float32)
    x = xt.float().cpu().numpy()
    got = serve.token_probs(xt, _dev(temperature, torch.float32), min_p=min_p)
    assert got.shape == (t, v) and got.dtype == torch.float32
    _check_probs(got, x, temperature, min_p)
    one = serve.token_probs(xt, 0.7, min_p=min_p)
    _check_probs(one, x, np.full(t, 0.7, np.float32), min_p)
    assert torch.equal(serve.token_probs(xt, 0.7, min_p=min_p), one)
    sp.check()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_probs_of_views_into_views(sp, serve, dtype):
    """Rows that begin at any address, results into rows that begin anywhere; nothing beside them is written.  The order in
    which a row is added up goes by its address, so that two views of one row are each held to the bound above, and a row
    alone or written elsewhere to the same numbers as among others."""
    g = np.random.default_rng(1)
    wide = _dev(g.standard_normal((6, 900)), torch.bfloat16 if dtype == "bf16" else torch.float32)
    for a in range(9):
        for v in (1, 17, 256, 801):
            x = wide[:, a:a + v]
            t = np.full(6, 0.5, np.float32)
            _check_probs(serve.token_probs(x.contiguous(), 0.5), x.float().cpu().numpy(), t, 0.0)
            want = serve.token_probs(x, 0.5)
            _check_probs(want, x.float().cpu().numpy(), t, 0.0)
            out = torch.full((6, 910), 7.0, device="cuda")
            for at in (a, a + 1):
                got = serve.token_probs(x, 0.5, out=out[:, at:at + v])
                assert torch.equal(got, want) and torch.equal(out[:, at:at + v], want)
                out[:, at:at + v] = 7.0
                assert (out == 7.0).all()
            assert torch.equal(serve.token_probs(x[2:3], 0.5), want[2:3])
    sp.check()


@pytest.mark.parametrize("v", [9, 40000])
def test_probs_of_special_rows(sp, serve, v):
    x = np.zeros((12, v), np.float32)
    x[1, 3] = np.nan
    x[2, 3] = np.inf
    x[3, :] = -np.inf
    x[4, :] = -np.inf
    x[4, v - 1] = -5
    x[5, :] = 3e38
    x[5, ::2] = -3e38
    x[6, 1:] = -np.inf
    x[7, :] = np.linspace(-1, 1, v)
    x[8, 2] = x[8, 7] = 1
    x[9, 3] = np.nan
    x[10, 4] = np.inf
    temperature = np.array([1, 1, 1, 1, 1e-30, 1, np.inf, 1e-38, -1, 0, 0, np.nan], np.float32)
    got = serve.token_probs(_dev(x, torch.float32), _dev(temperature, torch.float32))
    sp.check()
    _check_probs(got, x, temperature, 0.0)
    assert got[4, v - 1] == 1 and got[8, 2] == 1 and got[10, 4] == 1


def test_probs_of_no_rows_and_past_32_bits(sp, serve):
    assert serve.token_probs(torch.zeros((0, 5), device="cuda")).shape == (0, 5)
    t, v = 17000, 131071  # 2.2e9 entries, 8.9e9 bytes out
    x = torch.zeros((t, v), dtype=torch.bfloat16, device="cuda")
    x[-1, 5:] = -2.0
    x[t // 2, v - 1] = 11.0
    p = serve.token_probs(x)
    sp.check()
    for r in (0, t // 2, t - 1):
        _check_probs(p[r:r + 1], x[r:r + 1].float().cpu().numpy(), np.ones(1, np.float32), 0.0)


# ------------------------------------------------------------------ verification
def _verify_case(g, requests, most, vocab, given, prompts=True):
    """Random requests (idle ones, prompts before the drafts) over peaked distributions near one another."""
    drafts = g.integers(0, most + 1, requests)
    new = drafts + 1
    if prompts:
        new = new + np.where(g.random(requests) < 0.2, g.integers(1, 9, requests), 0)
        idle = g.random(requests) < 0.15
        new, drafts = np.where(idle, 0, new), np.where(idle, 0, drafts)
    if requests == 1:
        new, drafts = np.array([most + 1]), np.array([most])
    cu = np.concatenate([[0], np.cumsum(new)])
    t = int(cu[-1])
    x = 3 * g.standard_normal((t, vocab))
    p = np.exp(x) / np.exp(x).sum(-1, keepdims=True)
    y = x + 0.7 * g.standard_normal((t, vocab))
    q = np.exp(y) / np.exp(y).sum(-1, keepdims=True)
    ids = np.array([g.choice(vocab, p=q[j - 1]) if j else 0 for j in range(t)], np.int64).reshape(t)
    return p.astype(np.float32), q.astype(np.float32), ids, cu, drafts, g.random(t).astype(np.float32), g.random(requests).astype(np.float32)


def _call(serve, p, q, ids, cu, drafts, accept, sample, types=(torch.float32, torch.float32)):
    """The GPU's answer and the model's on the same numbers."""
    pt = _dev(p, types[0])
    qt = None if q is None else _dev(q, types[1])
    got = serve.verify_drafts(pt, _i64(ids), _i32(cu), _i32(drafts), _dev(accept, torch.float32), _dev(sample, torch.float32), draft_probs=qt)
    want = ref.verify(pt.float().cpu().numpy(), None if q is None else qt.float().cpu().numpy(), *([int(i) for i in a] for a in (ids, cu, drafts)),
                      list(np.float32(accept)), list(sample))
    return [a.tolist() for a in got], [list(map(int, w)) for w in want]


@pytest.mark.parametrize("requests,most,vocab", [(1, 0, 1), (1, 4, 3), (1, 4, 1000), (1, 40, 130), (3, 2, 32001), (7, 70, 50), (17, 5, 4095),
                                                 (40, 3, 257), (200, 4, 515), (400, 1, 64)])
@pytest.mark.parametrize("given", ["fp32", "bf16", "none"])
def test_verify(sp, serve, requests, most, vocab, given):
    g = np.random.default_rng(requests + most + vocab)
    p, q, *rest = _verify_case(g, requests, most, vocab, given)
    types = (torch.bfloat16 if vocab % 2 else torch.float32, torch.bfloat16 if given == "bf16" else torch.float32)
    got, want = _call(serve, p, None if given == "none" else q, *rest, types=types)
    assert got == want
    sp.check()


def test_verify_at_its_borders(sp, serve):
    """u q = p refuses; equal distributions keep everything; certain refusals and certain drafts; numbers at the ends."""
    p = np.array([[0.25, 0.25, 0.5, 0]] * 4, np.float32)
    q = np.array([[0.5, 0.25, 0.25, 0]] * 4, np.float32)
    below = np.nextafter(np.float32(0.5), np.float32(0))
    for ids, u, sample in (([9, 0, 2, 1], [0.5, 0, 0, 0], 0.0), ([9, 0, 2, 1], [below, 0.999, 0.99999994, 0], 0.99999994),
                           ([9, 3, 3, 3], [0.0, 0, 0, 0], 0.5), ([9, 2, 2, 3], [0.9, 0.9, 0.0, 0], 1.0), ([9, 0, 0, 0], [0, 0, 0, 0], -1.0),
                           ([9, 1, 0, 0], [0.99, 0.6, 0, 0], np.nan)):
        for draft in (q, p, None):
            got, want = _call(serve, p, draft, ids, [0, 4], [3], np.float32(u), np.float32([sample]))
            assert got == want, (ids, u)
    sp.check()


def test_verify_draws_every_entry_at_its_border(sp, serve):
    """Weights in 2^-10ths, so that floor(total u) falls on the first number of an entry, and one before it."""
    w = np.array([0, 3, 0, 5, 1, 0, 7, 0], np.float32) / 1024
    ups = np.concatenate([[0], np.cumsum(w)])
    us = np.concatenate([ups[:-1] / ups[-1], np.nextafter(np.float32(ups[1:] / ups[-1]), np.float32(0))]).astype(np.float32)
    p = np.tile(w, (len(us), 1))
    got, want = _call(serve, p, None, np.zeros(len(us)), np.arange(len(us) + 1), np.zeros(len(us)), np.zeros(len(us)), us)
    assert got == want and {1, 3, 4, 6} == set(got[2])
    # far entries of a long row, tiny weights, one after the other
    v = 70001
    p = np.zeros((6, v), np.float32)
    for r, at in enumerate((0, 1, 4095, 35000, 69999, 70000)):
        p[r, at] = 2.0 ** -40
    got, want = _call(serve, p, None, np.zeros(6), np.arange(7), np.zeros(6), np.zeros(6), np.float32([0, 0.5, 0.99999994] * 2))
    assert got == want == [[0] * 6, [0] * 6, [0, 1, 4095, 35000, 69999, 70000]]
    sp.check()


def test_verify_counts_what_is_no_probability_as_none(sp, serve):
    p = np.array([[np.nan, -1, 0.5, np.inf], [0, 0, 0, 0], [2.0, 0, 0, 1], [np.nan] * 4], np.float32)
    args = (np.zeros(4), np.arange(5), np.zeros(4), np.zeros(4), np.float32([0.5, 0.5, 0.4, 0.1]))
    got, want = _call(serve, p, None, *args)
    assert got == want and got[2] == [3, -1, 0, -1]
    with pytest.raises(sp.SpError):  # rows without any weight
        sp.check()
    got, want = _call(serve, p[:1], p[:1] * 0, np.zeros(1), [0, 1], [0], [0], [0.1])
    assert got == want and got[2] == [2]
    sp.check()


def test_verify_falls_back_where_nothing_is_left(sp, serve):
    """A refused draft with q >= p everywhere (probabilities that add up to less than 1)."""
    p = np.array([[0.1, 0.2, 0.3], [0.2, 0.2, 0.2]], np.float32)
    q = np.array([[0.2, 0.3, 0.4], [0.2, 0.2, 0.2]], np.float32)
    for u in (0.0, 0.2, 0.6, 0.99):
        got, want = _call(serve, p, q, [0, 0], [0, 2], [1], [0.9, 0], [u])
        assert got == want and got[0] == [0]
    sp.check()


@pytest.mark.parametrize("ids,cu,drafts", [([0, 9, 0], [0, 3], [2]), ([0, -1, 0], [0, 3], [2]), ([0, 1, 0], [0, 3], [3]),
                                           ([0, 1, 0], [0, 3], [-1]), ([0, 1, 0], [0, 4], [1]), ([0, 1, 0], [2, 1], [0]),
                                           ([0, 1, 0], [-1, 2], [1]), ([0, 1, 0], [-1, -1], [0])])
def test_verify_leaves_out_what_does_not_belong_together(sp, serve, ids, cu, drafts):
    p = np.full((3, 4), 0.25, np.float32)
    got, want = _call(serve, p, None, ids, cu, drafts, np.zeros(3), [0.3])
    assert got == want
    with pytest.raises(sp.SpError, match="INVALID_ARG"):
        sp.check()
    sp.check()


def test_verify_of_views_and_nothing(sp, serve):
    g = np.random.default_rng(3)
    p, q, ids, cu, drafts, accept, sample = _verify_case(g, 6, 3, 301, "fp32")
    t = p.shape[0]
    base = _call(serve, p, q, ids, cu, drafts, accept, sample)[0]
    args = (_i64(ids), _i32(cu), _i32(drafts), _dev(accept, torch.float32), _dev(sample, torch.float32))
    for a in range(5):
        pw, qw = torch.full((t, 320), 9.0, device="cuda"), torch.full((t, 400), 9.0, device="cuda")
        pw[:, a:a + 301], qw[:, 2 * a:2 * a + 301] = _dev(p, torch.float32), _dev(q, torch.float32)
        got = serve.verify_drafts(pw[:, a:a + 301], *args, draft_probs=qw[:, 2 * a:2 * a + 301])
        assert [x.tolist() for x in got] == base
    none = torch.zeros(0, device="cuda")
    got = serve.verify_drafts(torch.zeros((0, 5), device="cuda"), none.long(), _i32([0]), none.int(), none, none)
    assert [x.numel() for x in got] == [0, 0, 0]
    got = serve.verify_drafts(torch.zeros((0, 5), device="cuda"), none.long(), _i32([0, 0, 0]), _i32([0, 3]), none, torch.zeros(2, device="cuda"))
    assert [x.tolist() for x in got] == [[0, 0], [0, 0], [-1, -1]]
    sp.check()


def test_verify_past_32_bits(sp, serve):
    t, v = 18000, 131071
    p = torch.zeros((t, v), device="cuda")
    p[:, 7] = 0.5
    p[-1, v - 1] = 0.5
    ids = torch.full((t,), 7, device="cuda")
    got = serve.verify_drafts(p, ids, _i32([0, 3, t - 3, t]), _i32([2, 1, 2]), torch.zeros(t, device="cuda"), _dev([0.1, 0.1, 0.9], torch.float32))
    sp.check()
    assert [x.tolist() for x in got] == [[2, 1, 2], [0, 0, 0], [7, 7, v - 1]]


def test_accepted_tokens_have_the_targets_distribution(sp, serve):
    """Of 40000 requests with one draft each: how often each token comes first in the answer.  A count of mean n p has
    deviation at most sqrt(n p); five of them."""
    n, v = 40000, 8
    p = np.array([0.3, 0.05, 0.2, 0.1, 0.05, 0.0, 0.25, 0.05], np.float32)
    q = np.array([0.1, 0.3, 0.1, 0.1, 0.1, 0.1, 0.1, 0.1], np.float32)
    g = torch.Generator(device="cuda").manual_seed(0)
    pt, qt = _dev(np.tile(p, (2 * n, 1)), torch.float32), _dev(np.tile(q, (2 * n, 1)), torch.float32)
    ids = torch.multinomial(qt, 1, generator=g)[:, 0]
    cu = 2 * torch.arange(n + 1, device="cuda", dtype=torch.int32)
    for draft in (qt, None):
        a, r, nxt = serve.verify_drafts(pt, ids, cu, torch.ones(n, dtype=torch.int32, device="cuda"), torch.rand(2 * n, generator=g, device="cuda"),
                                        torch.rand(n, generator=g, device="cuda"), draft_probs=draft)
        first = torch.where(a == 1, ids[1::2], nxt)
        count = torch.bincount(first, minlength=v).double().cpu().numpy()
        assert (np.abs(count - n * p) <= 5 * np.sqrt(n * p) + 1e-6).all() and torch.equal(a + r, torch.ones_like(a))
    sp.check()


# ------------------------------------------------------------------ tokens taken back
def _batch(serve, g, b, page, width, hold=True):
    cached = g.integers(0, width * page + 1, b)
    pages_of = lambda n: -(-n // page)  # noqa: E731
    held = int(sum(pages_of(n) for n in cached))
    pages = held + 9
    order = g.permutation(pages)
    table = np.full((b, width), -1)
    at = 0
    for i, n in enumerate(cached):
        table[i, :pages_of(n)] = order[at:at + pages_of(n)]
        at += pages_of(n)
    batch = serve.Batch(serve.KvCache(pages, 1, 64, page), 1, b, 4, width)
    batch.cached.copy_(_i32(cached))
    batch.table.copy_(_i32(table.reshape(b, width)))
    batch.free[:9] = _i32(order[held:])
    batch.free_count.fill_(9)
    return batch, cached.tolist(), table.tolist(), order[held:].tolist()


@pytest.mark.parametrize("b,page,width", [(1, 16, 1), (1, 64, 300), (3, 16, 5), (64, 32, 20), (1000, 16, 6), (1024, 128, 2), (1025, 16, 4), (5000, 16, 3)])
@pytest.mark.parametrize("some", ["few", "any", "all", "none"])
def test_retract(sp, serve, b, page, width, some):
    g = np.random.default_rng(b + page)
    batch, cached, table, free = _batch(serve, g, b, page, width)
    drop = [int(min(c, {"few": g.integers(0, 5), "any": g.integers(0, c + 1), "all": c, "none": 0}[some])) for c in cached]
    lens, stack = ref.retract(cached, drop, table, free, page)
    before = batch.table.clone()
    for advance in (False, False, True):
        batch.retract(_i32(drop), advance=advance)
        assert batch.status.item() == 0 and batch.lens.tolist() == lens
        assert batch.next_count.item() == len(stack) and batch.free[:len(stack)].tolist() == stack
        assert batch.cached.tolist() == (lens if advance else cached) and torch.equal(batch.table, before)
    sp.check()


def test_retract_without_pages(sp, serve):
    batch, cached, _, _ = _batch(serve, np.random.default_rng(0), 5, 16, 3)
    kept = batch.free.clone()
    batch.retract(_i32([min(c, 17) for c in cached]), advance=True, allocate=False)
    assert batch.cached.tolist() == [c - min(c, 17) for c in cached]
    assert torch.equal(batch.free, kept) and batch.free_count.item() == 9
    sp.check()


@pytest.mark.parametrize("what", ["more", "negative", "length", "height", "stack"])
@pytest.mark.parametrize("advance", [False, True])
def test_retract_that_cannot_be(sp, serve, what, advance):
    batch, cached, _, _ = _batch(serve, np.random.default_rng(1), 6, 16, 4)
    drop, height = [0] * 6, 9
    i = int(np.argmax(cached))
    drop[i] = 17
    if what == "more":
        drop[i] = cached[i] + 1
    elif what == "negative":
        drop[2] = -1
    elif what == "length":
        cached[1] = 65
        batch.cached[1] = 65
    elif what == "height":
        height = -1
        batch.free_count.fill_(-1)
    else:
        height = batch.pages
        batch.free_count.fill_(height)
    kept = batch.free.clone()
    batch.status.fill_(4)  # what a plan said stays
    batch.retract(_i32([0] * 6) if what in ("more", "negative") else _i32(drop), advance=False)
    assert batch.status.item() == (4 if what in ("more", "negative") else 12)
    batch.status.zero_()
    batch.retract(_i32(drop), advance=advance)
    assert batch.status.item() == 8 and batch.lens.tolist() == cached == batch.cached.tolist()
    assert torch.equal(batch.free, kept) and batch.next_count.item() == height == batch.free_count.item()
    sp.check()


def test_a_step_planned_taken_back_and_planned_again(sp, serve):
    """Three requests grow, lose some of it, and grow again: every page is in one place."""
    page, width = 16, 8
    batch = serve.Batch(serve.KvCache(24, 1, 64, page), 1, 3, 64, width)
    g = np.random.default_rng(2)
    lens = [0, 0, 0]
    for step in range(60):
        new = [int(min(g.integers(0, 20), width * page - n)) for n in lens]
        if step % 7 == 6:
            new[step % 3] = -1
        batch.plan(_i32(new), advance=True)
        assert batch.status.item() == 0
        lens = [0 if a < 0 else n + a for n, a in zip(lens, new)]
        drop = [int(g.integers(0, max(a, 0) + 1)) for a in new]
        batch.retract(_i32(drop), advance=True)
        lens = [n - d for n, d in zip(lens, drop)]
        assert batch.cached.tolist() == lens and batch.status.item() == 0
        held = [p for b, n in enumerate(lens) for p in batch.table[b, :-(-n // page)].tolist()]
        free = batch.free[:batch.free_count.item()].tolist()
        assert sorted(held + free) == list(range(24))
    sp.check()


def test_the_three_in_a_graph_on_another_stream(sp, serve):
    g = np.random.default_rng(4)
    p, q, ids, cu, drafts, accept, sample = _verify_case(g, 5, 4, 1003, "fp32", prompts=False)
    t = p.shape[0]
    logits = _dev(np.log(p), torch.float32)
    draft, args = _dev(q, torch.float32), (_i64(ids), _i32(cu), _i32(drafts), _dev(accept, torch.float32), _dev(sample, torch.float32))
    batch = serve.Batch(serve.KvCache(50, 1, 64, 16), 1, 5, t, 8)
    new = _i32(np.diff(cu))

    def step():
        batch.plan(new, advance=True)
        probs = serve.token_probs(logits)
        a, r, n = serve.verify_drafts(probs, args[0], batch.cu_q, *args[2:], draft_probs=draft)
        batch.retract(r, advance=True)
        return probs, a, r, n

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        want = step()
    s.synchronize()
    lens = batch.cached.tolist()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for i in range(2, 5):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want))
        assert batch.cached.tolist() == [i * n for n in lens]
    sp.check()
