"""Serving operators on the GPU where the numbers of one call lie far apart.

Bounds are those of tests/test_gpu_serve.py.  A query row that is larger by a factor of 2^30 and more has one
key that takes all the weight (its scores are that far apart, their errors 2^-20 of them), so its own result
is that key's value, rounded once; and no row's bound depends on another's size."""
import numpy as np
import pytest

from paper_2405_03594_gb300 import synth
from tests import gpu_util as gu
from tests import serve_ref as ref
from tests.test_gpu_serve import Filled, _near, serve, sp  # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu


def _scaled(f, rows, by):
    """The queries of `rows` ((token, head) pairs) times `by`."""
    x = synth.bf16_to_f32(f.q)
    for t, h in rows:
        x[t, h] *= np.float32(by)
    f.q = synth.bf16_from_f32(x)
    f.qd = gu.bf16_to_dev(f.q)


@pytest.mark.parametrize("by", [2.0 ** 16, 2.0 ** 26, 2.0 ** 30, 2.0 ** 34, 2.0 ** 40, 2.0 ** 100])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("heads,kv,new", [(4, 1, [1, 1, 1]), (12, 1, [1, 1, 1]), (8, 2, [5, 3, 2]), (8, 2, [8, 7, 1]),
                                          (4, 1, [40, 3, 90])])
def test_a_row_of_large_queries_leaves_its_neighbours_alone(sp, serve, heads, kv, new, d, by):  # noqa: F811
    """One head of one token is scaled up, in every row tile that it shares: the other heads and tokens of the
    tile keep their results (8, 16, 24, 32 rows, and the kernel for many)."""
    g = np.random.default_rng(heads + sum(new))
    f = Filled(serve, g, [300, 40, 170], new, heads, kv, d, 32)
    _scaled(f, [(0, heads - 1), (new[0], 0), (sum(new) - 1, heads // 2)], by)
    y = f.cache.attend(f.qd, f.batch, max(new))
    sp.check()
    _near(y, f.want(), f.vmax())


@pytest.mark.parametrize("heads,kv,new", [(4, 1, [1, 1, 1]), (8, 2, [5, 3, 2]), (8, 2, [8, 7, 1]), (4, 1, [40, 3, 90])])
@pytest.mark.parametrize("d", [64, 128])
def test_queries_near_the_end_of_the_range(sp, serve, heads, kv, new, d):  # noqa: F811
    """Queries of 2^118 to 2^120: their scores are still fp32 numbers."""
    g = np.random.default_rng(3 * heads + sum(new))
    f = Filled(serve, g, [300, 40, 170], new, heads, kv, d, 16)
    _scaled(f, [(t, h) for t in range(sum(new)) for h in range(0, heads, 2)], 2.0 ** 118)
    y = f.cache.attend(f.qd, f.batch, max(new))
    sp.check()
    _near(y, f.want(), f.vmax())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("t,v", [(9, 130), (9, 1100), (9, 32000), (3, 131071), (700, 1500)])
def test_order_of_rows_that_are_not_finite(sp, serve, dtype, t, v):  # noqa: F811
    """All NaN (more of them than the kernel lists at a time, too), NaN at the first entries, among infinities:
    a NaN counts as the largest, equal ones go by rising index."""
    import torch

    g = np.random.default_rng(v)
    x = (2 * g.standard_normal((t, v))).astype(np.float32)
    x[0] = np.nan
    x[1, 0] = np.nan
    x[2, : v // 2] = np.inf
    if t > 3:
        x[3, 3:] = np.nan
        x[4, [0, 5, v - 1]] = np.nan
        x[4, [1, 7]] = np.inf
        x[5] = -np.inf
        x[6] = np.inf
        x[7], x[7, 0] = -np.inf, np.nan
    xd = torch.tensor(x, device=gu.dev())
    if dtype == "bf16":
        xd = xd.bfloat16()
        x = xd.float().cpu().numpy()
    for top in (1, 20, 64):
        ids = g.integers(0, v, t)
        lp, en, tl, ti = serve.token_logprobs(xd, torch.tensor(ids, device=gu.dev()), top)
        wl, we, wt, wi = ref.logprobs(x.astype(np.float64), ids, top)
        assert np.array_equal(ti.cpu().numpy(), wi), top
        for a, e in ((lp, wl), (en, we), (tl, wt)):
            assert np.array_equal(np.isnan(a.cpu().numpy()), np.isnan(e))
    sp.check()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("v", [40, 3001, 70000])
def test_zeros_of_either_sign(sp, serve, dtype, v):  # noqa: F811
    """-0 comes below +0, each by rising index; their log probabilities are the same."""
    import torch

    x = torch.full((3, v), -1.0)
    x[0, : v // 2] = -0.0
    x[0, 1:12:3] = 0.0
    x[1] = -0.0
    x[2] = 0.0
    lp, _, tl, ti = serve.token_logprobs(x.to(gu.dev()).to(torch.bfloat16 if dtype == "bf16" else torch.float32),
                                         torch.zeros(3, dtype=torch.int64, device=gu.dev()), 8)
    sp.check()
    assert ti.tolist() == [[1, 4, 7, 10, 0, 2, 3, 5], list(range(8)), list(range(8))]
    assert torch.equal(tl, lp[:, None].expand(3, 8))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("heads,kv,new,lens", [(8, 2, [1, 2], [700, 90]), (8, 2, [40, 3, 90], [700, 90, 100]),
                                               (4, 4, [300], [900])])
@pytest.mark.parametrize("offset", [50.0, 1000.0, -20000.0])
def test_keys_far_from_zero(sp, serve, heads, kv, new, lens, d, offset):  # noqa: F811
    """Keys whose entries all lie `offset` from zero, a thousand times their spread and more: their codes still
    tell them apart, with few and with many query rows.  The offset is multiplied by the queries' sum in fp32: with
    |sum(q)| < 100 and scale <= 1/8, a part of a score up to 2.5e5, rounded to 2^-24 of itself in each of three operations: at
    most 5e-2 of a weight, and 8e-3 of the norm for such errors at random (a third of them, over equal weights' halves)."""
    g = np.random.default_rng(int(abs(offset)))
    f = Filled(serve, g, lens, new, heads, kv, d, 32)
    n, s, m = f.rows[0]
    m += np.float16(offset)
    f.load()
    y = f.cache.attend(f.qd, f.batch, max(new))
    sp.check()
    w, got = f.want(), gu.bf16_from_dev(y)
    assert np.abs(got - w).max() <= (5e-2 if abs(offset) > 1e4 else 8e-3) * f.vmax() + 2.0 ** -8 * np.abs(w).max()
    assert np.linalg.norm(got - w) <= (8e-3 if abs(offset) > 1e4 else 2.5e-3) * np.linalg.norm(w)


@pytest.mark.parametrize("case", ["large_offset", "peaked", "equal", "scale"])
def test_distributions_of_many_rows(sp, serve, case):  # noqa: F811
    """The distributions that tests/test_gpu_serve.py has for few rows, for the kernel of many."""
    g = np.random.default_rng(12)
    f = Filled(serve, g, [700, 90], [70, 33], 8, 2, 128, 64, offset=50.0 if case == "large_offset" else 0.0)
    scale = {"peaked": 4.0, "scale": -0.02}.get(case)
    if case == "equal":
        for n, s, m in f.rows[:1]:
            n[:], s[~np.isnan(s)], m[~np.isnan(m)] = 3, 0.5, -1
        f.load()
    y = f.cache.attend(f.qd, f.batch, 70, scale=scale)
    sp.check()
    if case == "peaked":  # scores four times sqrt(128) as large: so are their errors
        w = f.want(scale)
        assert np.abs(gu.bf16_from_dev(y) - w).max() <= 0.2 * f.vmax()
        assert np.linalg.norm(gu.bf16_from_dev(y) - w) <= 1e-2 * np.linalg.norm(w)
    else:
        _near(y, f.want(scale), f.vmax())
