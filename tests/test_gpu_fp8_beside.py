"""Nothing beside the results of an 8-bit linear is written, where rows of y start at multiples of 16 bytes, and end anywhere."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m", [1, 8, 16, 33, 64, 65, 100, 300, 1000])
@pytest.mark.parametrize("n,stride", [(1, 8), (100, 104), (100, 112), (97, 104), (63, 72), (65, 128), (127, 136), (129, 144), (191, 200), (257, 264),
                                      (1001, 1016), (5003, 5016), (104, 112), (256, 264)])
@pytest.mark.parametrize("at", [0, 8])
def test_nothing_beside_rows_on_sixteen_bytes_is_written(m, n, stride, at):
    from paper_2405_03594_gb300 import fp8, sp

    g = torch.Generator(device="cuda").manual_seed(m + n)
    k = 640 if n < 1000 else 260
    x = torch.randn((m, k), generator=g, device="cuda").bfloat16()
    w = fp8.Fp8Matrix.from_dense((0.05 * torch.randn((n, k), generator=g, device="cuda")).bfloat16())
    want = w.linear(x)
    wide = torch.full((m + 2, at + stride), 7.0, dtype=torch.bfloat16, device="cuda")
    assert wide[1:, at:].data_ptr() % 16 == 0 and wide.stride(0) % 8 == 0
    for rows in (x, fp8.quantize_rows(x)):
        got = w.linear(rows, out=wide[1:m + 1, at:at + n])
        sp.check()
        assert torch.equal(got, want)
        wide[1:m + 1, at:at + n] = 7.0
        assert (wide == 7.0).all()


@pytest.mark.parametrize("n,m,k", [(12284, 512, 256), (22013, 4096, 200), (1003, 140, 9000)])  # wide tiles; tiles that are shared
def test_nothing_beside_large_results_is_written(n, m, k):
    from paper_2405_03594_gb300 import fp8, sp

    g = torch.Generator(device="cuda").manual_seed(n)
    x = torch.randn((m, k), generator=g, device="cuda").bfloat16()
    w = fp8.Fp8Matrix.from_dense((0.05 * torch.randn((n, k), generator=g, device="cuda")).bfloat16())
    want = w.linear(x)
    wide = torch.full((m + 2, (n + 15) // 8 * 8), 7.0, dtype=torch.bfloat16, device="cuda")
    got = w.linear(x, out=wide[1:m + 1, :n])
    sp.check()
    assert torch.equal(got, want)
    wide[1:m + 1, :n] = 7.0
    assert (wide == 7.0).all()


def test_two_layers_into_one_buffer():
    """Rows of 60 and of 68 columns side by side: the second stays as it is when the first is computed again."""
    from paper_2405_03594_gb300 import fp8, sp

    g = torch.Generator(device="cuda").manual_seed(0)
    x = torch.randn((200, 384), generator=g, device="cuda").bfloat16()
    a, b = (fp8.Fp8Matrix.from_dense((0.05 * torch.randn((n, 384), generator=g, device="cuda")).bfloat16()) for n in (60, 68))
    both = torch.empty((200, 128), dtype=torch.bfloat16, device="cuda")
    for _ in range(2):
        b.linear(x, out=both[:, 60:])
        a.linear(x, out=both[:, :60])
    sp.check()
    assert torch.equal(both, torch.cat([a.linear(x), b.linear(x)], 1))
