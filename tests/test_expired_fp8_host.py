"""The failure-path call of the 8-bit linears: its refusals, which return before any GPU work (CPU)."""


def test_expired_fp8_refusals():
    from paper_2405_03594_gb300 import sp

    a = sp.SpFp8LinearArgs()
    for n in ("w", "w_scale", "x", "y"):
        setattr(a, n, 1 << 20)
    a.w_stride, a.x_stride, a.y_stride, a.m, a.n, a.k = 112, 100, 50, 2, 50, 100
    call = lambda a, *b: sp._lib.sp_test_expired_fp8(a, 1 << 20, 1 << 30, *b, None)  # noqa: E731
    assert call(None, 0, 0, 0, 5) == 1
    for b in ((-1, 0, 0, 5), (0, -1, 0, 5), (0, 0, -1, 5), (0, 0, 0, 0), (0, 0, 0, 10001)):
        assert call(a, *b) == 1, b
    a.y += 1
    assert call(a, 0, 0, 0, 5) == 3
    a.y, a.m = 1 << 20, 0
    assert call(a, 0, 0, 0, 5) == 0
