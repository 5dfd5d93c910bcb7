"""Serving operators on the GPU at steps large enough that a warp or CTA takes several rows of work: the
loops over heads of the rotation and of the read, the log probabilities' CTAs of 128 threads.  Models and bounds
are those of tests/test_gpu_serve.py; the counts below are for 152 multiprocessors."""
import numpy as np
import pytest

from tests import gpu_util as gu
from tests.test_gpu_serve import _check_logprobs, serve, sp  # noqa: F401  (fixtures)
from tests.test_gpu_serve import test_norm_rope_and_cache_rows as _check_rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("t,h,kv,d,rot", [(1200, 33, 11, 128, 128), (1500, 33, 11, 128, 64), (4096, 33, 11, 128, 128),
                                          (3000, 30, 10, 64, 64), (5500, 30, 10, 64, 32), (4001, 17, 3, 64, 64),
                                          (2500, 5, 5, 128, 128)])
@pytest.mark.parametrize("normed,pairs", [(True, False), (False, True)])
def test_several_rows_of_heads_per_warp(sp, serve, t, h, kv, d, rot, normed, pairs):  # noqa: F811
    """2, 3, 8, 3, 6, 2 and 1 rows of heads per warp, the last ones partly filled; rows read back by 2 to 4 warps a slot."""
    _check_rows(sp, serve, t, h, kv, d, rot, normed, pairs)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("t,v,top", [(608, 9000, 1), (700, 9000, 20), (700, 8999, 64), (613, 4097, 64), (700, 40, 20),
                                     (640, 2047, 0)])
def test_logprobs_of_many_rows(sp, serve, dtype, t, v, top):  # noqa: F811
    """A CTA of 128 threads a row: the search for the best entries, by threads (up to four vectors each) and by
    whole warps, rows of equal entries (more of them than are listed at a time, too) and rows almost shut."""
    import torch

    g = np.random.default_rng(t + v)
    x = (3 * g.standard_normal((t, v))).astype(np.float32)
    x[1] = 0.75
    x[2] = -np.inf
    x[3], x[3, [0, v - 1]] = -np.inf, [1, 2]
    x[4, : v // 2] = x[4].max() + 1
    x[5] = np.round(x[5])
    x[6, 7] = np.nan
    ids = g.integers(0, v, t)
    ids[::7] = -1
    xd = torch.tensor(x, device=gu.dev())
    if dtype == "bf16":
        xd = xd.bfloat16()
        x = xd.float().cpu().numpy()
    x = np.where(x == 0, np.float32(0), x)  # (zeros of either sign are another test's)
    xd = torch.where(xd == 0, torch.zeros_like(xd), xd)
    _check_logprobs(serve, xd, x.astype(np.float64), ids, top)
    sp.check()
