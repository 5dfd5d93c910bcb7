"""Serving operators on the GPU against the plain models of tests/serve_ref.py.

Tables, norms, rotation and 4-bit rows are defined bit for bit, so they are compared for equality
(bf16 results of the rotation too).  Attention rounds once to bf16 (half a unit in the last place,
2^-9 of the value) after fp32 sums: a score is a sum of codes up to 143 times queries in 8 steps, off
by at most 8 * 2^-22 * 143 * sum|q| * s * scale <= 4e-3 for the inputs here (sum|q| < 250, s < 0.6,
scale <= 1/8), so a weight by 4e-3 of itself, and the average by at most 8e-3 of the largest |v|.
Errors are random, so the whole is held to the rounding: 2.5e-3 of the norm (one rounding: 1.7e-3).
Log probabilities: fp32 sums of up to 131071 terms by threads of at most 300, and one logarithm:
2e-6 of max(1, |value|)."""
import numpy as np
import pytest

from paper_2405_03594_gb300 import synth
from tests import gpu_util as gu
from tests import serve_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sp():
    from paper_2405_03594_gb300 import sp as _sp

    return _sp


@pytest.fixture(scope="module")
def serve():
    from paper_2405_03594_gb300 import serve as _s

    return _s


def _i32(a):
    import torch

    return torch.tensor(np.asarray(a, np.int32), device=gu.dev())


def _i64(a):
    import torch

    return torch.tensor(np.asarray(a, np.int64), device=gu.dev())


def _bf(a):
    return gu.bf16_to_dev(synth.bf16_from_f32(np.asarray(a, np.float32)))


# ------------------------------------------------------------------ tables
def _plan_case(serve, g, b, page, width, tokens, group=1):
    """A batch with random lengths and its model."""
    pages_of = lambda n: -(-n // page)  # noqa: E731
    cached = g.integers(0, width * page // 2 + 1, b)
    cached[g.random(b) < 0.2] = 0
    held = int(sum(pages_of(n) for n in cached))
    pages = held + int(b * width // 2) + 1
    order = g.permutation(pages)
    table = np.full((b, width), -1)
    at = 0
    for i, n in enumerate(cached):
        table[i, :pages_of(n)] = order[at:at + pages_of(n)]
        at += pages_of(n)
    free = order[held:]
    cache = serve.KvCache(pages, 1, 64, page)
    batch = serve.Batch(cache, group, b, tokens, width)
    batch.cached.copy_(_i32(cached))
    batch.table.copy_(_i32(table.reshape(b, width)))
    batch.free[:len(free)] = _i32(free)
    batch.free_count.fill_(len(free))
    return batch, ref.Tables(cached.tolist(), table.tolist(), free.tolist(), page, tokens)


def _check_plan(batch, want):
    lens, cu, slots, pos, table, free, status = want
    assert batch.status.item() == status
    assert batch.lens.tolist() == list(lens)
    assert batch.cu_q.tolist() == cu
    assert batch.slots.tolist() == slots and batch.positions.tolist() == pos
    assert batch.table.tolist() == [list(r) for r in table]
    assert batch.next_count.item() == len(free) and batch.free[:len(free)].tolist() == list(free)


@pytest.mark.parametrize("b,page,width,tokens", [(1, 16, 1, 1), (1, 64, 9, 300), (3, 16, 5, 40), (64, 32, 20, 64),
                                                 (1000, 16, 6, 20000), (1024, 128, 2, 4096), (1025, 16, 4, 4097),
                                                 (5000, 16, 3, 9000)])
@pytest.mark.parametrize("ends", [False, True])
def test_plan_steps(sp, serve, b, page, width, tokens, ends):
    """A step that can be planned again, then the step taken, and one more after it."""
    g = np.random.default_rng(b + page)
    batch, model = _plan_case(serve, g, b, page, width, tokens, group=3)
    for _ in range(2):
        new = np.minimum(g.integers(0, max(2, 2 * tokens // (3 * b)), b), width * page - np.array(model.cached))
        while new.sum() > tokens:
            new[np.argmax(new)] //= 2
        if ends:
            new[g.random(b) < 0.2] = -1
        want = model.step(new.tolist())
        assert want[6] == 0
        for _ in range(2):
            batch.plan(_i32(new))
            _check_plan(batch, want)
        batch.plan(_i32(new), advance=True)
        _check_plan(batch, want)
        assert batch.cached.tolist() == want[0]
        model.cached, model.table, model.free = list(want[0]), want[4], want[5]
    sp.check()


@pytest.mark.parametrize("what", ["pages", "width", "tokens", "cached"])
@pytest.mark.parametrize("advance", [False, True])
def test_plan_that_does_not_fit(sp, serve, what, advance):
    g = np.random.default_rng(5)
    batch, model = _plan_case(serve, g, 7, 16, 8, 60)
    new = [3, 0, 5, 1, -1, 2, 7]
    if what == "pages":
        batch.free_count.fill_(0)
        model.free, new = [], [20, 20, 20, 0, 0, 0, 0]
    elif what == "width":
        model.max_tokens = batch.tokens
        new[2] = 8 * 16 - model.cached[2] + 1
        batch.cached[0] = model.cached[0] = 0
    elif what == "tokens":
        new = [9] * 7
    else:
        batch.cached[3] = model.cached[3] = -1
    want = list(model.step(new)) if what != "cached" else [model.cached, [0] * 8, [-1] * 60, [0] * 60, model.table, model.free, 8]
    assert want[6] != 0
    batch.plan(_i32(new), advance=advance)
    _check_plan(batch, want)
    sp.check()


def test_plan_complete_table_empty_batch_and_graph(sp, serve):
    import torch

    g = np.random.default_rng(6)
    batch, model = _plan_case(serve, g, 9, 16, 8, 50)
    full = g.permutation(9 * 8).reshape(9, 8)
    batch.table.copy_(_i32(full))
    model.table = full.tolist()
    new = [1, 0, 5, 30, 0, 0, 2, 1, 1]
    free, count = batch.free.clone(), batch.free_count.item()
    batch.plan(_i32(new), allocate=False)
    lens, cu, slots, pos, _, _, status = model.step(new, allocate=False)
    assert (batch.lens.tolist(), batch.cu_q.tolist(), batch.slots.tolist(), batch.positions.tolist()) == (lens, cu, slots, pos)
    assert batch.table.tolist() == full.tolist() and batch.status.item() == status == 0
    assert torch.equal(batch.free, free) and batch.free_count.item() == count
    empty = serve.Batch(serve.KvCache(1, 1, 64, 16), 1, 0, 0, 1)
    empty.plan(_i32([]))
    assert empty.cu_q.tolist() == [0] and empty.status.item() == 0
    # growing by one token per replay
    batch, model = _plan_case(serve, g, 5, 16, 30, 5)
    one = _i32([1] * 5)
    gr = torch.cuda.CUDAGraph()
    with torch.cuda.graph(gr):
        batch.plan(one, advance=True)
    for _ in range(40):
        want = model.step([1] * 5)
        gr.replay()
        torch.cuda.synchronize()
        _check_plan(batch, want)
        model.cached, model.table, model.free = list(want[0]), want[4], want[5]
    sp.check()


# ------------------------------------------------------------------ norms, rotation, 4-bit rows
def _qkv(g, t, h, kv, d, special=False):
    x = g.standard_normal((t, h + 2 * kv, d)).astype(np.float32)
    x[:, h:h + kv] *= np.exp(g.standard_normal((kv, d))).astype(np.float32)
    if special and t >= 6:
        x[1, h + kv:] = 3.0            # a constant row
        x[2, h + kv:] *= np.float32(1e-9)  # scales below fp16's range
        x[3, h + kv:] *= np.float32(1e6)   # above it
        x[4, h + kv, 5] = np.inf
        x[5, h, 7] = np.nan
    return synth.bf16_from_f32(x)


def _angles(g, rows, rot):
    a = g.random((rows, rot // 2)) * 7
    return np.concatenate([np.cos(a), np.sin(a)], 1).astype(np.float32)


@pytest.mark.parametrize("t,h,kv,d,rot", [(1, 32, 32, 128, 128), (1, 1, 1, 64, 64), (7, 5, 1, 128, 64), (33, 32, 8, 128, 128),
                                          (257, 6, 3, 64, 32), (1500, 8, 8, 64, 64), (700, 32, 4, 128, 16), (40, 7, 7, 128, 0)])
@pytest.mark.parametrize("normed,pairs", [(False, False), (True, False), (True, True), (False, True)])
def test_norm_rope_and_cache_rows(sp, serve, t, h, kv, d, rot, normed, pairs):
    import torch

    g = np.random.default_rng(t + rot)
    bits = _qkv(g, t, h, kv, d, special=True)
    x = synth.bf16_to_f32(bits)
    rows, page = 300, 16
    cs = _angles(g, rows, rot)
    pos = g.integers(0, rows, t)
    qw, kw = (synth.bf16_from_f32((1 + 0.4 * g.standard_normal((2, d))).astype(np.float32))) if normed else (None, None)
    pages = -(-t // page) + 2
    slots = g.permutation(pages * page)[:t]
    if t > 8:
        slots[8] = -1
    dev = gu.bf16_to_dev(bits.reshape(t, -1)).view(t, h + 2 * kv, d)
    q, k, v = dev[:, :h], dev[:, h:h + kv], dev[:, h + kv:]
    cache = serve.KvCache(pages, kv, d, page)
    cache.data.fill_(0xff)
    kw_ = dict(eps=1e-6, pairs=pairs, q_weight=None if qw is None else gu.bf16_to_dev(qw),
               k_weight=None if kw is None else gu.bf16_to_dev(kw))
    table = torch.tensor(cs, device=gu.dev()) if rot else torch.zeros((rows, 0), device=gu.dev())
    qo = cache.append(q, k, v, _i32(pos), _i64(slots), table, **kw_)
    q2, k2 = serve.qk_norm_rope(q, k, _i32(pos), table, **kw_)
    with np.errstate(all="ignore"):
        want = []
        for y, w in ((x[:, :h], qw), (x[:, h:h + kv], kw)):
            if w is not None:
                y = ref.norm(y, synth.bf16_to_f32(w), 1e-6)
            want.append(ref.rotate(y, cs[pos, :rot // 2], cs[pos, rot // 2:], pairs))
    for got, y in ((qo, want[0]), (q2, want[0]), (k2, want[1])):
        a = synth.bf16_to_f32(gu.bf16_bits_from_dev(got))
        e = ref.bf16(y)[0]
        nan = np.isnan(y)
        assert np.array_equal(np.isnan(a), nan) and np.array_equal(a[~nan], e[~nan])
    got = ref.unpack(cache.data.cpu().numpy(), pages, kv, page, d)
    kept = slots >= 0
    untouched = np.ones((pages, kv, page), bool)
    for i, y in ((0, want[1]), (1, x[:, h + kv:])):
        n, s, m = ref.quantize(y)
        pg, at = slots // page, slots % page
        gn = got[3 * i][pg, :, at]
        gs, gm = got[3 * i + 1][pg, :, at], got[3 * i + 2][pg, :, at]
        assert np.array_equal(gn[kept], n[kept])
        assert np.array_equal(gs[kept], s[kept])
        assert np.array_equal(np.isnan(gm[kept]), np.isnan(m[kept]))
        f = kept[:, None] & ~np.isnan(m)
        assert np.array_equal(gm[f], m[f])
        untouched[pg[kept], :, at[kept]] = False
        assert (got[3 * i][untouched] == 15).all()
    # and read back
    rk, rv = cache.read(_i64(slots))
    for got_, y in ((rk, want[1]), (rv, x[:, h + kv:])):
        n, s, m = ref.quantize(y)
        e = ref.bf16(ref.values(n, s, m).astype(np.float32))[0]
        e[~kept] = 0
        a = synth.bf16_to_f32(gu.bf16_bits_from_dev(got_))
        nan = np.isnan(e)
        assert np.array_equal(np.isnan(a), nan) and np.array_equal(a[~nan], e[~nan])
    sp.check()


def test_rope_bad_indices_are_left_out_and_recorded(sp, serve):
    g = np.random.default_rng(1)
    t, h, kv, d, page = 4, 2, 2, 64, 16
    x = gu.bf16_to_dev(_qkv(g, t, h, kv, d).reshape(t, -1)).view(t, h + 2 * kv, d)
    import torch

    cs = torch.tensor(_angles(g, 5, d), device=gu.dev())
    cache = serve.KvCache(2, kv, d, page)
    cache.data.fill_(7)
    cache.append(x[:, :h], x[:, h:h + kv], x[:, h + kv:], _i32([0] * 4), _i64([-1, 32, 1 << 40, -(1 << 50)]), cs)
    with pytest.raises(sp.SpError) as e:
        sp.check()
    assert e.value.code == 1 and (cache.data == 7).all()
    for pos in ([0, 0, 5, 0], [0, -1, 0, 0]):
        a, _ = serve.qk_norm_rope(x[:, :h], x[:, h:h + kv], _i32(pos), cs)
        b, _ = serve.qk_norm_rope(x[:, :h], x[:, h:h + kv], _i32([0] * 4), cs)
        with pytest.raises(sp.SpError):
            sp.check()
        assert torch.equal(a, b)
    k, v = cache.read(_i64([0, 32, -5, 31]))
    assert not k[1:3].any() and not v[1:3].any() and k[0].any()
    with pytest.raises(sp.SpError):
        sp.check()
    sp.check()
    q, k = serve.qk_norm_rope(x[:0, :h], x[:0, h:h + kv], _i32([]), cs)  # no tokens
    assert q.shape == (0, h, d) and k.shape == (0, kv, d)


# ------------------------------------------------------------------ attention
class Filled:
    """A cache whose every slot holds random rows, and the requests of a batch over it."""

    def __init__(self, serve, g, lens, new, heads, kv, d, page, offset=0.0):
        import torch

        need = [-(-n // page) for n in lens]
        width = max(max(need, default=1), 1)
        pages = sum(need) + 2
        x = g.standard_normal((2, pages, kv, page, d)).astype(np.float32)
        x[0] *= np.exp(0.4 * g.standard_normal((kv, 1, d))).astype(np.float32)
        x[1] += offset + g.standard_normal((kv, 1, d)).astype(np.float32)
        self.rows = [ref.quantize(x[i]) for i in range(2)]
        order = g.permutation(pages)
        table = np.full((len(lens), width), -1)
        at = 0
        for b, n in enumerate(need):
            table[b, :n] = order[at:at + n]
            at += n
            if lens[b] % page:  # slots that no token was written to
                for i in range(2):
                    for par in self.rows[i][1:]:
                        par[table[b, n - 1], :, lens[b] % page:] = np.nan
        self.lens, self.new, self.table, self.page, self.kv, self.d = lens, new, table, page, kv, d
        self.cache = serve.KvCache(pages, kv, d, page)
        self.batch = serve.Batch(self.cache, heads, len(lens), sum(new), width)
        self.load()
        self.batch.table.copy_(_i32(table))
        self.batch.cached.copy_(_i32(np.array(lens) - np.array(new)))
        self.batch.plan(_i32(new), allocate=False)
        assert self.batch.status.item() == 0
        self.q = synth.bf16_from_f32((1.5 * g.standard_normal((sum(new), heads, d))).astype(np.float32))
        self.qd = gu.bf16_to_dev(self.q)
        torch.cuda.synchronize()

    def load(self):
        import torch

        self.cache.data.copy_(torch.from_numpy(ref.pack(*self.rows[0], *self.rows[1])))

    def want(self, scale=None):
        scale = 1 / np.sqrt(self.d) if scale is None else scale
        q = synth.bf16_to_f32(self.q).astype(np.float64)
        kv = [ref.values(*r) for r in self.rows]
        out, at = [], 0
        for b, (n, a) in enumerate(zip(self.lens, self.new)):
            pg = self.table[b, :-(-n // self.page)]
            k, v = (y[pg].transpose(0, 2, 1, 3).reshape(-1, self.kv, self.d)[:n] for y in kv)
            out.append(ref.attend(q[at:at + a], k, v, scale))
            at += a
        return np.concatenate(out) if out else np.zeros(q.shape)

    def vmax(self):
        return np.nanmax(np.abs(ref.values(*self.rows[1])))


def _near(got, want, vmax, what=""):
    y = gu.bf16_from_dev(got)
    assert np.array_equal(np.isnan(y), np.isnan(want)), what
    f = ~np.isnan(want)
    err = np.abs(y - want)[f]
    assert (err <= 2.0 ** -8 * np.abs(want[f]) + 8e-3 * vmax).all(), (what, err.max())
    n = np.linalg.norm(want[f])
    assert np.linalg.norm(err) <= 2.5e-3 * n + 1e-30, (what, np.linalg.norm(err) / n)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("heads,kv", [(1, 1), (4, 4), (8, 1), (6, 2), (7, 1), (16, 1)])
def test_decode_lengths(sp, serve, d, page, heads, kv):
    """One token each at lengths around tiles, pages and shares."""
    g = np.random.default_rng(page + heads)
    lens = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 300, 777]
    f = Filled(serve, g, lens, [1] * len(lens), heads, kv, d, page)
    y = f.cache.attend(f.qd, f.batch, 1)
    sp.check()
    _near(y, f.want(), f.vmax())


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("heads,kv,new", [(4, 4, [2, 1, 0, 3, 8]), (8, 2, [5, 8, 1, 0, 4]), (32, 8, [3, 6, 2, 8, 1]),
                                          (3, 3, [40, 1, 17, 0, 100]), (8, 1, [9, 33, 2, 64, 0]), (64, 1, [2, 1, 5, 3, 1]),
                                          (14, 2, [70, 1, 128, 3, 200])])
def test_several_new_tokens(sp, serve, d, heads, kv, new):
    """Causal among the new tokens, requests without any, and requests that hold nothing else."""
    g = np.random.default_rng(sum(new) + heads)
    lens = [n + a for n, a in zip([100, 0, 50, 333, 0], new)]
    f = Filled(serve, g, lens, new, heads, kv, d, 32)
    y = f.cache.attend(f.qd, f.batch, max(new))
    sp.check()
    _near(y, f.want(), f.vmax())


@pytest.mark.parametrize("lens,new,heads,kv", [([20000], [1], 8, 1), ([9000, 3, 0, 700], [1, 1, 0, 1], 4, 4),
                                               ([5000], [4], 32, 8), ([4097], [1], 32, 32),
                                               ([5000], [40], 32, 8), ([3000, 90, 0], [300, 20, 0], 8, 8)])
def test_long_contexts_are_split_and_joined(sp, serve, lens, new, heads, kv):
    g = np.random.default_rng(lens[0])
    f = Filled(serve, g, lens, new, heads, kv, 128, 64)
    import torch

    ws = torch.zeros(f.cache.workspace_size(), dtype=torch.uint8, device=gu.dev())
    ys = [f.cache.attend(f.qd, f.batch, max(new), workspace=ws) for _ in range(3)]
    sp.check()
    _near(ys[0], f.want(), f.vmax())
    assert torch.equal(ys[0], ys[1]) and torch.equal(ys[0], ys[2])
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    assert not ws[:32 * sms].any()  # the arrival counters: ready for the next call, of sp_linear too


@pytest.mark.parametrize("lens,new,heads,kv,d", [([600, 4000, 20, 300, 140], [600, 34, 0, 300, 129], 64, 32, 64),
                                                 ([1500], [1500], 32, 32, 64), ([700] * 3, [700, 650, 513], 32, 32, 128),
                                                 ([40 + 8 * i for i in range(33)], [40] * 33, 8, 8, 64)])
def test_more_pairs_of_tiles_than_multiprocessors(sp, serve, lens, new, heads, kv, d):
    """Prompts of different and of equal lengths, whose work is taken in order of its size; more than 32 of them."""
    g = np.random.default_rng(sum(lens))
    f = Filled(serve, g, lens, new, heads, kv, d, 16)
    y = f.cache.attend(f.qd, f.batch, max(new))
    sp.check()
    _near(y, f.want(), f.vmax())


def test_many_requests(sp, serve):
    g = np.random.default_rng(3)
    lens = g.integers(1, 300, 500).tolist()
    f = Filled(serve, g, lens, [1] * 500, 4, 2, 64, 16)
    y = f.cache.attend(f.qd, f.batch, 1)
    sp.check()
    _near(y, f.want(), f.vmax())


@pytest.mark.parametrize("case", ["large_offset", "peaked", "equal", "scale"])
def test_distributions(sp, serve, case):
    """Values far from zero, one key that takes all, keys that are all the same, another scale."""
    g = np.random.default_rng(11)
    f = Filled(serve, g, [700, 90], [1, 2], 8, 2, 128, 64, offset=50.0 if case == "large_offset" else 0.0)
    scale = None
    if case == "peaked":
        scale = 4.0
    if case == "scale":
        scale = -0.02
    if case == "equal":
        for n, s, m in f.rows[:1]:
            n[:], s[~np.isnan(s)], m[~np.isnan(m)] = 3, 0.5, -1
        f.load()
    y = f.cache.attend(f.qd, f.batch, 2, scale=scale)
    sp.check()
    if case == "peaked":  # scores four times sqrt(128) as large: so are their errors
        w = f.want(scale)
        assert np.abs(gu.bf16_from_dev(y) - w).max() <= 0.2 * f.vmax()
        assert np.linalg.norm(gu.bf16_from_dev(y) - w) <= 1e-2 * np.linalg.norm(w)
    else:
        _near(y, f.want(scale), f.vmax())


def test_nan_rows_reach_only_who_sees_them(sp, serve):
    g = np.random.default_rng(12)
    new = [6, 1, 40]
    f = Filled(serve, g, [106, 50, 90], new, 4, 2, 128, 16)
    for i, (b, at, head) in enumerate([(0, 103, 0), (2, 70, 1)]):  # the fourth new token's key, a value
        row = f.rows[i]
        row[1][f.table[b, at // 16], head, at % 16] = 0
        row[2][f.table[b, at // 16], head, at % 16] = np.nan
    f.load()
    y = f.cache.attend(f.qd, f.batch, 40)
    sp.check()
    w = f.want()
    assert np.isnan(w).any() and not np.isnan(w).all()
    _near(y, w, f.vmax())


@pytest.mark.parametrize("heads,kv,new", [(8, 2, [1, 2, 1]), (8, 2, [6, 1, 8]), (4, 1, [40, 3, 90])])
def test_queries_that_are_not_finite_or_of_far_scales(sp, serve, heads, kv, new):
    """An infinity or NaN makes NaN of its own row alone; rows a factor of 2^40 apart do not disturb each
    other (the queries' scaling is a power of two per row, or of the rows of a tile)."""
    g = np.random.default_rng(21)
    f = Filled(serve, g, [300, 40, 170], new, heads, kv, 64, 32)
    x = synth.bf16_to_f32(f.q)
    x[0, 1] *= np.float32(2.0 ** -20)
    x[-1, 0] *= np.float32(2.0 ** -40)
    x[0, 0, 3] = np.inf
    x[1, 2, 60] = np.nan
    x[-1, 1] = 0
    f.q = synth.bf16_from_f32(x)
    y = f.cache.attend(gu.bf16_to_dev(f.q), f.batch, max(new))
    sp.check()
    x[0, 0, 3] = x[1, 2, 60] = 0
    f.q = synth.bf16_from_f32(x)
    w = f.want()
    w[0, 0] = w[1, 2] = np.nan
    got = gu.bf16_from_dev(y)
    assert np.isnan(got[0, 0]).all() and np.isnan(got[1, 2]).all()
    _near(y, w, f.vmax())


@pytest.mark.parametrize("kv,d,new", [(1, 128, 1), (2, 64, 2), (1, 128, 40), (1, 64, 300)])
def test_flat_attention_over_a_long_context(sp, serve, kv, d, new):
    """Weights that are nearly equal over 60000 keys: an average of many values, far below each of them."""
    g = np.random.default_rng(22)
    f = Filled(serve, g, [60000], [new], 4 * kv, kv, d, 128)
    f.q = synth.bf16_from_f32((0.02 * g.standard_normal((new, 4 * kv, d))).astype(np.float32))
    f.qd = gu.bf16_to_dev(f.q)
    y = f.cache.attend(f.qd, f.batch, new)
    sp.check()
    rows = [0, new - 1]
    f.q, f.lens, f.new = f.q[rows], [60000], [new]
    q = synth.bf16_to_f32(f.q).astype(np.float64)
    pg = f.table[0]
    k, v = (ref.values(*r)[pg].transpose(0, 2, 1, 3).reshape(-1, kv, d)[:60000] for r in f.rows)
    want = np.concatenate([ref.attend(q[i:i + 1], k[:60000 - new + r + 1], v[:60000 - new + r + 1], d ** -0.5)
                           for i, r in enumerate(rows)])
    got = gu.bf16_from_dev(y)[rows]
    # means of 60000 values of size 1 about their channels' offsets: the offsets dominate
    assert np.linalg.norm(got - want) <= 2.5e-3 * np.linalg.norm(want)
    assert np.abs(got - want).max() <= 2.0 ** -8 * np.abs(want).max() + 1e-3


def test_strided_queries_and_output(sp, serve):
    import torch

    g = np.random.default_rng(13)
    f = Filled(serve, g, [60, 5, 300], [3, 1, 2], 6, 3, 64, 16)
    wide = torch.full((6, 10, 64), float("nan"), dtype=torch.bfloat16, device=gu.dev())
    wide[:, 2:8] = f.qd
    out = torch.full((8, 9, 64), 7.0, dtype=torch.bfloat16, device=gu.dev())
    f.cache.attend(wide[:, 2:8], f.batch, 3, out=out[:6, 1:7])
    sp.check()
    _near(out[:6, 1:7].contiguous(), f.want(), f.vmax())
    out[:6, 1:7] = 7
    assert (out == 7).all()


def test_rows_behind_the_last_token_and_bad_tables(sp, serve):
    import torch

    g = np.random.default_rng(14)
    f = Filled(serve, g, [60, 5, 300], [3, 1, 2], 6, 3, 64, 16)
    q = torch.cat([f.qd, torch.full((4, 6, 64), float("nan"), dtype=torch.bfloat16, device=gu.dev())])
    out = torch.full_like(q, 7.0)
    f.cache.attend(q, f.batch, 3, out=out)
    sp.check()
    _near(out[:6], f.want(), f.vmax())
    assert (out[6:] == 7).all()
    # a page that does not exist takes no part, and is recorded
    good = f.batch.table.clone()
    for bad in (-1, f.cache.pages, 1 << 30):
        f.batch.table[2, 3] = bad
        y = f.cache.attend(f.qd, f.batch, 3)
        with pytest.raises(sp.SpError) as e:
            sp.check()
        assert e.value.code == 1 and torch.equal(y[:4], out[:4])
        f.batch.table.copy_(good)
    # more new tokens than the call was told of: nothing is written for that request
    out.fill_(7)
    f.cache.attend(f.qd, f.batch, 2, out=out[:6])
    with pytest.raises(sp.SpError):
        sp.check()
    assert (out[:3] == 7).all() and not (out[3:6] == 7).all()
    many = Filled(serve, g, [50, 20], [40, 1], 2, 2, 64, 16)
    y = torch.full_like(many.qd, 7.0)
    many.cache.attend(many.qd, many.batch, 1, out=y)
    with pytest.raises(sp.SpError):
        sp.check()
    assert (y[:40] == 7).all() and not (y[40] == 7).all()
    # lengths that the tables were not planned for
    f.batch.lens[0] = 500
    f.cache.attend(f.qd, f.batch, 3)
    with pytest.raises(sp.SpError):
        sp.check()
    f.batch.lens[0] = 60
    y = f.cache.attend(f.qd, f.batch, 3)
    sp.check()
    _near(y, f.want(), f.vmax())


def test_blocks_beyond_4_gib(sp, serve):
    """Slots and blocks whose offsets pass 32 bits."""
    import torch

    g = np.random.default_rng(15)
    page, kv, d = 128, 8, 128
    pages = (5 << 30) // (page * kv * (d + 8))
    f = Filled(serve, g, [300, 129], [1, 2], 16, kv, d, page)
    big = serve.KvCache(pages, kv, d, page)
    n = f.cache.data.numel()
    big.data[-n:] = f.cache.data
    first = pages - f.cache.pages
    f.batch.table.add_(first * (f.batch.table >= 0).int())
    y = big.attend(f.qd, f.batch, 2)
    sp.check()
    _near(y, f.want(), f.vmax())
    slots = (first + 1) * page + torch.arange(4, device=gu.dev())
    k, v = big.read(slots)
    k0, v0 = f.cache.read(slots - first * page)
    assert torch.equal(k, k0) and torch.equal(v, v0)
    x = torch.randn((4, 3 * kv, d), device=gu.dev()).bfloat16()
    cs = torch.tensor(_angles(g, 5, d), device=gu.dev())
    for c, s in ((big, slots), (f.cache, slots - first * page)):
        c.append(x[:, :kv], x[:, kv:2 * kv], x[:, 2 * kv:], _i32([0, 1, 2, 3]), s, cs)
    assert torch.equal(big.data[-n:], f.cache.data)
    del big


def test_on_another_stream_and_in_a_graph(sp, serve):
    import torch

    g = np.random.default_rng(16)
    f = Filled(serve, g, [2000, 5, 300], [1, 1, 1], 8, 2, 128, 64)
    want = f.cache.attend(f.qd, f.batch, 1)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    a = torch.empty_like(want)
    f.cache.attend(f.qd, f.batch, 1, out=a, stream=s)
    with torch.cuda.stream(s):
        b = f.cache.attend(f.qd, f.batch, 1)
    gr = torch.cuda.CUDAGraph()
    with torch.cuda.graph(gr):
        c = f.cache.attend(f.qd, f.batch, 1)
    gr.replay()
    gr.replay()
    torch.cuda.synchronize()
    sp.check()
    assert torch.equal(a, want) and torch.equal(b, want) and torch.equal(c, want)


# ------------------------------------------------------------------ log probabilities
def _check_logprobs(serve, logits, x, ids, top):
    got = serve.token_logprobs(logits, _i64(ids), top)
    lp, en, tl, ti = ref.logprobs(x, ids, top)
    for a, e in zip(got[:2] + got[2:3], (lp, en, tl)):
        a = a.cpu().numpy().astype(np.float64)
        assert np.array_equal(np.isnan(a), np.isnan(e))
        inf = np.isinf(e)
        assert np.array_equal(a[inf], e[inf])
        f = np.isfinite(e)
        assert np.isfinite(a[f]).all() and (np.abs(a - e)[f] <= 2e-6 * np.maximum(1, np.abs(e[f]))).all(), np.abs(a - e)[f].max()
    if top:
        assert np.array_equal(got[3].cpu().numpy(), ti)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("t,v,top", [(1, 1, 1), (3, 7, 7), (2, 15, 0), (1, 64, 64), (5, 1000, 5), (1, 32000, 20), (2, 32001, 64),
                                     (40, 50003, 3), (400, 999, 64), (3, 131071, 20), (1, 131071, 0)])
def test_logprobs(sp, serve, dtype, t, v, top):
    import torch

    g = np.random.default_rng(v + top)
    x = (3 * g.standard_normal((t, v))).astype(np.float32)
    ids = g.integers(0, v, t)
    ids[0] = -1 if t > 2 else ids[0]
    xd = torch.tensor(x, device=gu.dev())
    if dtype == "bf16":
        xd = xd.bfloat16()
        x = xd.float().cpu().numpy()
    _check_logprobs(serve, xd, x.astype(np.float64), ids, top)
    sp.check()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("v", [130, 32000, 70001])
def test_logprobs_special_rows(sp, serve, dtype, v):
    """Rows of equal entries, shut vocabularies, nothing at all, infinities, NaN, a far maximum."""
    import torch

    g = np.random.default_rng(v)
    x = (2 * g.standard_normal((12, v))).astype(np.float32)
    x[0] = 1.5
    x[1] = -np.inf
    x[2], x[2, [3, v // 2, v - 1]] = -np.inf, [1, 2, 1]
    x[3, 17] = np.nan
    x[4, [5, 80]] = np.inf
    x[5, 9] = 1e4
    x[6] = 0
    x[6, ::2] = -0.0
    x[7, :] = -3e38
    x[7, 4] = 3e38
    x[8, 10:90] = 50
    x[9] = np.where(g.random(v) < 0.5, -np.inf, x[9])
    x[10, [v - 1, 0]] = 30
    ids = g.integers(0, v, 12)
    ids[2], ids[5] = v // 2, 9
    xd = torch.tensor(x, device=gu.dev())
    if dtype == "bf16":
        xd = xd.bfloat16()
        x = xd.float().cpu().numpy()
    x = x.astype(np.float64)
    # equal zeros of either sign are one number to the model and two to the kernel's order: +0 first
    y = x.copy()
    y[6] = np.where(np.signbit(x[6]), -1e-300, 0)
    got = serve.token_logprobs(xd, _i64(ids), 20)
    _, _, _, ti = ref.logprobs(y, ids, 20)
    assert np.array_equal(got[3].cpu().numpy()[[0, 1, 2, 6, 7, 8, 9, 10, 11]], ti[[0, 1, 2, 6, 7, 8, 9, 10, 11]])
    lp, en, tl, _ = ref.logprobs(x, ids, 20)
    for a, e in zip(got[:3], (lp, en, tl)):
        a = a.cpu().numpy().astype(np.float64)
        with np.errstate(over="ignore"):
            e = e.astype(np.float32).astype(np.float64)  # (-6e38 is no float32)
        assert np.array_equal(np.isnan(a), np.isnan(e))
        f = np.isfinite(e)
        assert np.array_equal(a[~f & ~np.isnan(e)], e[~f & ~np.isnan(e)])
        assert (np.abs(a - e)[f] <= 2e-6 * np.maximum(1, np.abs(e[f]))).all()
    sp.check()


def test_logprobs_strides_alignment_and_bad_ids(sp, serve):
    import torch

    g = np.random.default_rng(1)
    for dtype in (torch.bfloat16, torch.float32):
        wide = torch.tensor(2 * g.standard_normal((9, 5000)), device=gu.dev()).to(dtype)
        for off, v in ((1, 4321), (3, 4001), (7, 8), (5, 2)):
            x = wide[:, off:off + v]
            _check_logprobs(serve, x, x.double().cpu().numpy(), g.integers(0, v, 9), min(v, 5))
    sp.check()
    x = wide[:2, :100]
    lp, _ = serve.token_logprobs(x, _i64([100, 1 << 40]))
    assert lp.isnan().all()
    with pytest.raises(sp.SpError) as e:
        sp.check()
    assert e.value.code == 1
    lp, en = serve.token_logprobs(wide[:0], _i64([]))
    assert lp.shape == (0,) and en.shape == (0,)


def test_python_checks(serve):
    import torch

    c = serve.KvCache(2, 2, 64, 16)
    q = torch.zeros((3, 4, 64), dtype=torch.bfloat16, device=gu.dev())
    k = q[:, :2]
    cs = torch.zeros((4, 64), device=gu.dev())
    pos, slots = _i32([0, 1, 2]), _i64([0, 1, 2])
    bad = [dict(q=q.float()), dict(q=q[:, :, :32]), dict(k=k[:2]), dict(v=k[:, :1]), dict(v=k.transpose(0, 1)),
           dict(positions=pos.long()), dict(positions=pos[:2]), dict(slots=slots.int()), dict(cos_sin=cs.double()),
           dict(q_weight=cs[0]), dict(out=q[:2])]
    for b in bad:
        kw = {**dict(q=q, k=k, v=k, positions=pos, slots=slots, cos_sin=cs), **b}
        with pytest.raises(ValueError):
            c.append(**kw)
    with pytest.raises(ValueError):
        serve.Batch(c, 3, 1, 1, 1)
    with pytest.raises(ValueError):
        serve.KvCache(2, 2, 64, 16, data=torch.zeros(5, dtype=torch.uint8, device=gu.dev()))
    b = serve.Batch(c, 4, 1, 3, 1)
    with pytest.raises(ValueError):
        b.plan(_i64([1]))
    with pytest.raises(ValueError):
        serve.KvCache(2, 2, 64, 32).attend(q, b, 1)
    with pytest.raises(ValueError):
        serve.token_logprobs(cs, _i32([0, 0, 0, 0]))
