"""The failure path of the 8-bit linears on the GPU, with nothing faulted, trapped or hung: one role's bounded wait is made to
expire (a shared-memory barrier that nothing completes and no copy targets), at first or with copies and products on their way.
The others find their waits expired in turn; the launch must end by itself and write nothing outside of y, sp_check must report
SP_ERR_TIMEOUT once, the workspace's counters must be at zero, and the next calls must be right."""
import time

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sp():
    from paper_2405_03594_gb300 import sp as _sp

    return _sp


@pytest.fixture(scope="module")
def fp8():
    from paper_2405_03594_gb300 import fp8 as _f

    return _f


class Case:
    def __init__(self, fp8, m, n, k, pad=8):
        g = torch.Generator(device="cuda").manual_seed(m + n + k)
        self.x = torch.randn((m, k), generator=g, device="cuda").bfloat16()
        self.w = fp8.Fp8Matrix.from_dense((0.05 * torch.randn((n, k), generator=g, device="cuda")).bfloat16())
        self.wide = torch.empty((m + 2, (n + pad + 7) // 8 * 8 + (pad & 1)), dtype=torch.bfloat16, device="cuda")
        self.ws = torch.zeros(max(256, self.w.workspace_size(m)), dtype=torch.uint8, device="cuda")
        self.m, self.n, self.k = m, n, k
        self.want = self.w.linear(self.x, workspace=self.ws)

    def args(self, sp):
        a = sp.SpFp8LinearArgs()
        a.w, a.w_scale, a.w_stride = *self.w._where, self.w._stride
        a.x, a.x_stride, a.y, a.y_stride = self.x.data_ptr(), self.k, self.wide[1:].data_ptr(), self.wide.stride(0)
        a.m, a.n, a.k = self.m, self.n, self.k
        return a

    def expire(self, sp, cta, warp, block, wait_ms=5):
        """Whether the warp gave up; checks what has to hold either way."""
        self.wide.fill_(7.0)
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        code = sp._lib.sp_test_expired_fp8(self.args(sp), self.ws.data_ptr(), self.ws.numel(), cta, warp, block, wait_ms, sp._stream())
        assert code == 0
        try:
            sp.check()
            gave_up = False
        except sp.SpError as e:
            assert e.code == 6  # SP_ERR_TIMEOUT
            gave_up = True
        assert time.perf_counter() - t0 < 2.0
        sp.check()  # reported once
        sms = torch.cuda.get_device_properties(0).multi_processor_count
        if self.ws.numel() > 256:
            assert not self.ws[:32 * sms].any(), (cta, warp, block)
        y = self.wide[1:self.m + 1, :self.n]
        if not gave_up:
            assert torch.equal(y, self.want)
        beside = self.wide.clone()
        beside[1:self.m + 1, :self.n] = 7.0
        assert (beside == 7.0).all(), (cta, warp, block)
        return gave_up

    def right(self, sp):
        for _ in range(2):
            assert torch.equal(self.w.linear(self.x, workspace=self.ws), self.want)
        sp.check()


# warps: epilogue 0-3, producer 4, products 5, quantisers 6-9 (where x is quantised on chip: up to 8 rows)
@pytest.mark.parametrize("m,n,k", [(1, 300, 4096), (8, 300, 4096), (1, 20000, 1024), (3, 20000, 1024), (12, 300, 4096), (16, 20000, 1024), (5, 130, 100)])
def test_a_role_of_the_kernel_for_few_tokens_gives_up(sp, fp8, m, n, k):
    """Clusters of eight with four blocks each, or a CTA with eight, three more than it holds; and a single block."""
    c = Case(fp8, m, n, k)
    roles = (0, 3, 4, 5, 6, 9) if m <= 8 else (0, 3, 4, 5)
    for warp in roles:
        for cta in (0, 1):
            if n > 128 * (cta + 1) or k > 128:
                assert c.expire(sp, cta, warp, 0), (cta, warp)
        for block in (1, 3, 6):
            assert c.expire(sp, 0, warp, block) == (block < (1 if k == 100 else 4 if n == 300 else 8)), (warp, block)
        c.right(sp)
    assert not c.expire(sp, 100000, 0, 0) and not c.expire(sp, 0, 10, 0) and not c.expire(sp, 0, 0, 1000)
    c.right(sp)


# warps: producer 0 (both CTAs of a pair), products 1 (the first), epilogue 4-11; 2 and 3 have no role
@pytest.mark.parametrize("m,n,k,pad", [(100, 1000, 9000, 8), (100, 1001, 9000, 9), (100, 7000, 2000, 8), (300, 100, 640, 9), (40960, 100, 640, 8), (256, 100, 5000, 8)])
def test_a_role_of_the_kernel_for_many_tokens_gives_up(sp, fp8, m, n, k, pad):
    """Tiles that pairs share, tiles of one pair with more blocks than it holds, and several tiles to a pair."""
    c = Case(fp8, m, n, k, pad)
    for cta in (0, 1, 3):
        for warp in (0, 1, 4, 7, 11):
            some = 0
            for block in (0, 1, 3, 9):
                some += c.expire(sp, cta, warp, block)
            assert (some >= 1) == (warp != 1 or cta % 2 == 0), (cta, warp)
        c.right(sp)
    assert not c.expire(sp, 0, 2, 0) and not c.expire(sp, 100000, 0, 0) and not c.expire(sp, 1, 1, 0)
    c.right(sp)


def test_expired_fp8_argument_checks(sp, fp8):
    c = Case(fp8, 3, 100, 200)
    call = lambda c, *a: sp._lib.sp_test_expired_fp8(c.args(sp), c.ws.data_ptr(), c.ws.numel(), *a, sp._stream())  # noqa: E731
    for a in ((-1, 0, 0, 5), (0, -1, 0, 5), (0, 0, -1, 5), (0, 0, 0, 0), (0, 0, 0, 10001)):
        assert call(c, *a) == 1, a
    assert call(Case(fp8, 20, 100, 200), 0, 0, 0, 5) == 2  # 17 rows to 64: not compiled
    assert call(Case(fp8, 4096, 4096, 512), 0, 0, 0, 5) == 2  # wider tiles
    sp.check()
