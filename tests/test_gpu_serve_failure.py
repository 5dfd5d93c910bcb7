"""The failure path of the attention kernels on the GPU, with nothing faulted, trapped or hung: one warp's
bounded wait is made to expire (a shared-memory barrier that nothing completes and no copy targets).  The
launch must end by itself, sp_check must report SP_ERR_TIMEOUT once, and the workspace must be as the next
calls need it: its counters at zero, their results those of a call before."""
import ctypes

import numpy as np
import pytest

from tests import gpu_util as gu
from tests.test_gpu_serve import Filled, serve, sp  # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu


def _args(sp, f, max_new, out):  # noqa: F811
    b, h, d = f.batch, f.qd.shape[1], f.d
    return sp.SpAttendArgs(f.qd.data_ptr(), out.data_ptr(), h * d, h * d, ctypes.pointer(f.cache._c), b.table.data_ptr(),
                           b.lens.data_ptr(), b.cu_q.data_ptr(), b.work.data_ptr(), f.qd.shape[0], b.requests, b.width, h,
                           max_new, d ** -0.5, 0)


def _expire(sp, f, max_new, ws, cta, warp, wait_ms=5):  # noqa: F811
    """Whether the warp gave up."""
    import torch

    out = torch.empty_like(f.qd)
    code = sp._lib.sp_test_expired_attend(_args(sp, f, max_new, out), ws.data_ptr(), ws.numel(), cta, warp, wait_ms,
                                          torch.cuda.current_stream().cuda_stream)
    assert code == 0
    try:
        sp.check()
    except sp.SpError as e:
        assert e.code == 6  # SP_ERR_TIMEOUT
        sp.check()  # reported once
        return True
    return False


@pytest.mark.parametrize("lens,new,heads,kv,page", [([100 + 37 * i % 500 for i in range(40)], [1] * 40, 8, 2, 16),
                                                    ([20000], [1], 8, 1, 64), ([5000, 40, 3000], [4, 1, 3], 8, 1, 32)])
def test_a_warp_that_gives_up_leaves_the_counters_as_they_were(sp, serve, lens, new, heads, kv, page):  # noqa: F811
    """Segments that begin and end in the midst of CTAs: every one is counted by all CTAs that share it."""
    import torch

    g = np.random.default_rng(len(lens))
    f = Filled(serve, g, lens, new, heads, kv, 64, page)
    ws = torch.zeros(f.cache.workspace_size(), dtype=torch.uint8, device=gu.dev())
    want = f.cache.attend(f.qd, f.batch, max(new), workspace=ws)
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    gave_up = 0
    for cta in range(0, sms, 5):
        for warp in (0, 1, 4, 7, 11):
            gave_up += _expire(sp, f, max(new), ws, cta, warp)
            assert not ws[:32 * sms].any(), (cta, warp)
    assert gave_up >= 20
    for _ in range(2):
        assert torch.equal(f.cache.attend(f.qd, f.batch, max(new), workspace=ws), want)
    sp.check()


@pytest.mark.parametrize("lens,new,heads,kv,page", [([3000, 50, 400], [300, 1, 90], 8, 2, 64), ([900], [700], 32, 32, 16),
                                                    ([5000], [40], 4, 1, 128)])
@pytest.mark.parametrize("warp", [0, 5, 8, 10, 11, 12, 13, 14, 15])
def test_a_role_of_the_kernel_for_many_rows_gives_up(sp, serve, lens, new, heads, kv, page, warp):  # noqa: F811
    """Each role (rows, codes to operands, products, copies; the last warp has none): the others find their waits
    expired in turn, the CTA ends, and the counters are at zero."""
    import time

    import torch

    g = np.random.default_rng(sum(lens))
    f = Filled(serve, g, lens, new, heads, kv, 64, page)
    ws = torch.zeros(f.cache.workspace_size(), dtype=torch.uint8, device=gu.dev())
    want = f.cache.attend(f.qd, f.batch, max(new), workspace=ws)
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    sp.check()
    gave_up = 0  # (which CTAs find work is their race; of 14 shares, perhaps none of these)
    for cta in range(0, sms, 8):
        t0 = time.perf_counter()
        gave_up += _expire(sp, f, max(new), ws, cta, warp)
        assert time.perf_counter() - t0 < 2.0
        assert not ws[:32 * sms].any(), cta
    assert gave_up == 0 if warp == 15 else gave_up >= 1 or sum(new) == 40
    for _ in range(2):
        assert torch.equal(f.cache.attend(f.qd, f.batch, max(new), workspace=ws), want)
    sp.check()


def test_expired_attend_argument_checks(sp, serve):  # noqa: F811
    import torch

    f = Filled(serve, np.random.default_rng(0), [50], [1], 2, 2, 64, 16)
    ws = torch.zeros(f.cache.workspace_size(), dtype=torch.uint8, device=gu.dev())
    out = torch.empty_like(f.qd)
    call = lambda max_new, *a: sp._lib.sp_test_expired_attend(_args(sp, f, max_new, out), ws.data_ptr(), ws.numel(), *a, None)  # noqa: E731
    for a in ((-1, 0, 5), (0, -1, 5), (0, 0, 0), (0, 0, 10001)):
        assert call(1, *a) == 1, a
    assert call(12, 0, 0, 5) == 2  # 12 rows: not compiled
    assert sp._lib.sp_test_expired_attend(_args(sp, f, 1, out), ws.data_ptr(), 16, 0, 0, 5, None) == 8
    assert not _expire(sp, f, 1, ws, 1000, 0)  # no such CTA
    sp.check()
