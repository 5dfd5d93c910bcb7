"""Serving operators on the GPU where the numbers of one call lie far apart.

Bounds are those of tests/test_gpu_serve.py.  A query row that is larger by a factor of 2^30 and more has one
key that takes all the weight (its scores are that far apart, their errors 2^-20 of them), so its own result
is that key's value, rounded once; and no row's bound depends on another's size."""
import numpy as np
import pytest

from paper_2405_03594_gb300 import synth
from tests import gpu_util as gu
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
