"""8-bit quantisation and linears on the GPU.

Codes and scales are defined bit for bit and compared for equality with the model of tests/drafts_ref.py.

The product is compared with the codes' values multiplied in 64 bits.  Products of two e4m3 numbers are exact in fp32;
a block's 128 of them are added in the tensor core, each addition off by at most a unit in the last place of fp32 (truncation),
2^-23 of the sum of magnitudes A so far; the scales' product, its product with the block's sum, and the sum over the
blocks round 2 + blocks times by 2^-24 of A.  At the end comes one rounding to bf16, 2^-8 of the value.  So
    |y - exact| <= 2^-8 |exact| + (128 + blocks + 2) 2^-23 A."""
import numpy as np
import pytest
import torch

from paper_2405_03594_gb300 import synth
from tests import drafts_ref as ref
from tests import gpu_util as gu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sp():
    from paper_2405_03594_gb300 import sp as _sp

    return _sp


@pytest.fixture(scope="module")
def fp8():
    from paper_2405_03594_gb300 import fp8 as _f

    return _f


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _x(m, k, g):
    x = torch.randn((m, k), generator=g, device="cuda") * torch.randn((k,), generator=g, device="cuda").exp_()
    return x.to(torch.bfloat16)


def _w(n, k, g):
    return (0.02 * torch.randn((n, k), generator=g, device="cuda") * torch.randn((n, 1), generator=g, device="cuda").exp_()).to(torch.bfloat16)


def _check(y, xq, w, rows=None):
    """y of quantised rows xq and the Fp8Matrix w."""
    blocks = -(-w.k // 128)
    y, q, s = y.double(), xq.codes.double(), xq.scale.double()
    if rows is not None:
        y, q, s = y[rows], q[rows], s[rows]
    want, most = torch.zeros_like(y), torch.zeros_like(y)
    sw = w.scale.double()
    for b in range(blocks):
        at = slice(128 * b, min(128 * (b + 1), w.k))
        qw = w.codes[:, at].double()
        f = s[:, b, None] * sw[:, b].repeat_interleave(128)[None, :w.n]
        want += (q[:, at] @ qw.T) * f
        most += (q[:, at].abs() @ qw.abs().T) * f
    off = (y - want).abs() - (2.0 ** -8 * want.abs() + (128 + blocks + 2) * 2.0 ** -23 * most)
    assert torch.isfinite(y).all() and off.max() <= 0, (off.max(), (y - want).norm() / want.norm())
    return (y - want).norm() / want.norm()


# ------------------------------------------------------------------ quantisation
@pytest.mark.parametrize("m,k", [(1, 1), (1, 128), (3, 7), (5, 129), (2, 256), (33, 1000), (130, 385), (64, 4096), (7, 11008)])
def test_rows_are_quantised_bit_for_bit(sp, fp8, m, k):
    g = np.random.default_rng(m * k)
    x = g.standard_normal((m, k)) * np.exp(3 * g.standard_normal((m, 1)))
    x[g.random((m, k)) < 0.01] *= 50
    x[m // 2, :] *= 0
    bits = synth.bf16_from_f32(x.astype(np.float32))
    q, s = ref.quantize(synth.bf16_to_f32(bits), 1)
    got = fp8.quantize_rows(gu.bf16_to_dev(bits))
    sp.check()
    assert np.array_equal(got.scale.cpu().numpy(), s)
    assert np.array_equal(got.codes.double().cpu().numpy(), q)


@pytest.mark.parametrize("n,k", [(1, 1), (128, 128), (129, 127), (3, 1000), (300, 257), (1000, 5)])
def test_weights_are_quantised_bit_for_bit(sp, fp8, n, k):
    g = np.random.default_rng(n + k)
    w = g.standard_normal((n, k)) * np.exp(g.standard_normal((n, 1)))
    w[: n // 3] *= 0
    bits = synth.bf16_from_f32(w.astype(np.float32))
    q, s = ref.quantize(synth.bf16_to_f32(bits), 128)
    got = fp8.Fp8Matrix.from_dense(gu.bf16_to_dev(bits))
    sp.check()
    assert np.array_equal(got.scale.cpu().numpy(), s)
    assert np.array_equal(got.codes.double().cpu().numpy(), q)
    assert np.array_equal(got.dense().cpu().numpy(), q.astype(np.float32) * np.repeat(np.repeat(s, 128, 0)[:n], 128, 1)[:, :k])


def test_quantisation_at_the_ends_of_the_range(sp, fp8):
    x = torch.zeros((8, 256), device="cuda")
    x[0, :3] = torch.tensor([3.3e38, -1.0, 1e30])
    x[1, :3] = torch.tensor([1e-38, -1e-39, 1e-40])
    x[2, 5] = float("inf")
    x[3, 200] = float("-inf")
    x[4, 7] = float("nan")
    x[5, :] = 2.0 ** -126
    x[6, 0], x[6, 1:128] = 448.0, torch.arange(127, device="cuda") / 8
    bits = gu.bf16_bits_from_dev(x.to(torch.bfloat16))
    q, s = ref.quantize(synth.bf16_to_f32(bits), 1)
    got = fp8.quantize_rows(x.to(torch.bfloat16))
    sp.check()
    assert np.array_equal(got.scale.cpu().numpy(), s, equal_nan=True)
    # (of blocks with a NaN or an infinity the codes are not defined, but what comes of them is: below)
    fine = np.repeat(np.isfinite(s), 128, 1)
    assert np.array_equal(np.where(fine, got.codes.double().cpu().numpy(), 0), np.where(fine, q, 0))


def test_quantisation_of_views(sp, fp8):
    g = _gen(1)
    wide = _x(9, 700, g)
    for view in (wide[:, 3:300], wide[:, 8:264], wide[::2, 16:529], wide[1:2, 1:200], wide[:, :1]):
        a, b = fp8.quantize_rows(view), fp8.quantize_rows(view.contiguous())
        assert torch.equal(a.codes.view(torch.uint8), b.codes.view(torch.uint8)) and torch.equal(a.scale, b.scale)
        a, b = fp8.Fp8Matrix.from_dense(view), fp8.Fp8Matrix.from_dense(view.contiguous())
        assert torch.equal(a.codes.view(torch.uint8), b.codes.view(torch.uint8)) and torch.equal(a.scale, b.scale)
    sp.check()


# ------------------------------------------------------------------ the product
SIZES = [(1, 1, 1), (1, 128, 128), (1, 4096, 4096), (2, 130, 5), (3, 127, 129), (8, 5000, 300), (15, 256, 2049), (16, 300, 384),
         (17, 129, 257), (31, 1000, 1000), (33, 127, 1000), (48, 2000, 513), (64, 1000, 640), (65, 129, 129), (100, 70, 4000),
         (127, 333, 100), (128, 1024, 1024), (129, 257, 385), (200, 3000, 128), (256, 512, 2048), (257, 700, 1111), (299, 5003, 1999),
         (511, 1100, 700), (600, 4096, 2000), (1000, 900, 11008), (1025, 130, 600), (2049, 2100, 130),
         (512, 12288, 256), (300, 12301, 390), (1030, 7000, 129), (70, 30000, 640)]


@pytest.mark.parametrize("m,n,k", SIZES)
def test_linear(sp, fp8, m, n, k):
    g = _gen(m + n + k)
    x, w = _x(m, k, g), fp8.Fp8Matrix.from_dense(_w(n, k, g))
    xq = fp8.quantize_rows(x)
    y = w.linear(x)
    sp.check()
    assert y.dtype == torch.bfloat16 and y.shape == (m, n)
    _check(y, xq, w)
    assert torch.equal(w.linear(xq), y) and torch.equal(w.linear(x), y)  # bitwise repeatable, either way
    sp.check()


def test_linear_m0(sp, fp8):
    w = fp8.Fp8Matrix.from_dense(_w(40, 50, _gen(0)))
    x = torch.empty((0, 50), dtype=torch.bfloat16, device="cuda")
    assert w.linear(x).shape == (0, 40) and w.linear(fp8.quantize_rows(x)).shape == (0, 40)


@pytest.mark.parametrize("m", [1, 20, 130, 700])
def test_linear_of_views_into_views(sp, fp8, m):
    g = _gen(m)
    wide, big = _x(m, 900, g), _w(500, 900, g)
    out = torch.full((m + 2, 640), 7.0, dtype=torch.bfloat16, device="cuda")
    for a, n in ((5, 300), (8, 257), (0, 128)):
        x = wide[:, a:a + 600]
        w = fp8.Fp8Matrix.from_dense(big[:n, a:a + 600])
        out.fill_(7.0)
        got = w.linear(x, out=out[1:m + 1, 3:3 + n])
        assert got.data_ptr() == out[1:, 3:].data_ptr()
        assert torch.equal(got, w.linear(x.contiguous()))
        left = out.clone()
        left[1:m + 1, 3:3 + n] = 7.0
        assert (left == 7.0).all()  # nothing beside it is written
    sp.check()


def test_matrix_of_given_codes(sp, fp8):
    """Codes with rows off 16 bytes are copied; others stay where they are, and later changes of them count."""
    g = _gen(3)
    base = fp8.Fp8Matrix.from_dense(_w(200, 300, g))
    x = _x(9, 300, g)
    y = base.linear(x)
    tight = base.codes.contiguous()
    assert tight.stride(0) == 300
    assert torch.equal(fp8.Fp8Matrix(tight, base.scale).linear(x), y)
    assert torch.equal(fp8.Fp8Matrix(tight.view(torch.uint8), base.scale).linear(x), y)
    wide = torch.zeros((200, 512), dtype=torch.uint8, device="cuda")
    wide[:, 16:316] = tight.view(torch.uint8)
    same = fp8.Fp8Matrix(wide[:, 16:316], base.scale)
    assert same._codes.data_ptr() == wide.data_ptr() + 16
    assert torch.equal(same.linear(x), y)
    wide.zero_()
    assert not same.linear(x).any()
    one = fp8.Fp8Matrix(tight[:1], base.scale[:1])
    assert torch.equal(one.linear(x), y[:, :1])
    off = fp8.Fp8Matrix(wide[:, 3:303], base.scale)
    assert not off.linear(x).any()
    sp.check()


@pytest.mark.parametrize("m", [3, 70, 300])
def test_numbers_that_are_not_finite_stay_in_their_rows(sp, fp8, m):
    g = _gen(m)
    k, n = 500, 300
    x, wd = _x(m, k, g), _w(n, k, g)
    clean = fp8.Fp8Matrix.from_dense(wd).linear(x)
    x[1, 130], x[2, 499] = float("nan"), float("inf")
    wd[140, 3] = float("nan")
    y = fp8.Fp8Matrix.from_dense(wd).linear(x)
    sp.check()
    assert torch.isnan(y[1:3]).all() and torch.isnan(y[:, 128:256]).all()
    rows = [i for i in range(m) if i not in (1, 2)]
    for at in (slice(0, 128), slice(256, 300)):
        assert torch.equal(y[rows, at], clean[rows, at])


@pytest.mark.parametrize("m", [2, 150])
def test_scales_at_the_ends_of_the_range(sp, fp8, m):
    """Rows and weights of very different size: every block's sum is scaled on its own."""
    g = _gen(9)
    x = (_x(m, 512, g).float() * torch.tensor([1e30, 1e-30, 1.0, 1e-4], device="cuda").repeat_interleave(128)).to(torch.bfloat16)
    w = (_w(130, 512, g).float() * torch.tensor([1e-30, 1e30, 1.0, 1e4], device="cuda").repeat_interleave(128)).to(torch.bfloat16)
    w = fp8.Fp8Matrix.from_dense(w)
    _check(w.linear(x), fp8.quantize_rows(x), w)
    sp.check()


def test_linear_past_32_bits(sp, fp8):
    """Codes, then results, of more than 2^32 bytes."""
    g = _gen(4)
    n, k = 140000, 32768
    codes = torch.randint(0, 120, (n, k), generator=g, dtype=torch.uint8, device="cuda")
    w = fp8.Fp8Matrix(codes, torch.rand((1094, 256), generator=g, device="cuda"))
    x = _x(3, k, g)
    y, xq = w.linear(x), fp8.quantize_rows(x)
    sp.check()
    last = fp8.Fp8Matrix(codes[-96:], w.scale[-1:])
    assert 140000 - 96 == 128 * 1093
    _check(y[:, -96:], xq, last)
    _check(y[:, :128], xq, fp8.Fp8Matrix(codes[:128], w.scale[:1]))
    del codes, w, last, y
    m, n = 70000, 33000
    x, w = _x(m, 128, g), fp8.Fp8Matrix.from_dense(_w(n, 128, g))
    y = w.linear(x)
    sp.check()
    _check(y, fp8.quantize_rows(x), w, rows=torch.tensor([0, 1, 255, 32767, 65535, 65536, m - 129, m - 1], device="cuda"))


# ------------------------------------------------------------------ streams, graphs, workspaces
def test_linear_on_another_stream_and_with_a_given_workspace(sp, fp8):
    g = _gen(5)
    x, w = _x(90, 700, g), fp8.Fp8Matrix.from_dense(_w(900, 700, g))
    y = w.linear(x)
    ws = torch.zeros(w.workspace_size(90), dtype=torch.uint8, device="cuda")
    assert torch.equal(w.linear(x, workspace=ws), y)
    with pytest.raises(sp.SpError, match="WORKSPACE"):
        w.linear(x, workspace=ws[:-256])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        y2 = torch.empty_like(y)
    w.linear(x, out=y2, stream=s)
    s.synchronize()
    assert torch.equal(y2, y)
    sp.check()


@pytest.mark.parametrize("m", [1, 50, 300])
def test_linears_in_graphs_that_share_a_stream(sp, fp8, m):
    """Two captured graphs and eager calls, replayed in turn: each with the numbers that are in its input now."""
    g = _gen(6)
    a, b = fp8.Fp8Matrix.from_dense(_w(1300, 520, g)), fp8.Fp8Matrix.from_dense(_w(520, 1300, g))
    x = _x(m, 520, g)
    b.linear(a.linear(x))
    torch.cuda.synchronize()
    graphs, outs = [], []
    for _ in range(2):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            outs.append(b.linear(a.linear(x)))
        graphs.append(gr)
    for i in range(4):
        x.copy_(_x(m, 520, g))
        want = b.linear(a.linear(x))
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[i % 2], want)
    sp.check()


def test_a_weight_written_just_before_the_call(sp, fp8):
    """The quantiser and the product back to back, again and again: no call sees codes from before."""
    g = _gen(7)
    codes = torch.zeros((4096, 1024), dtype=torch.uint8, device="cuda")
    scale = torch.zeros((32, 8), device="cuda")
    w = fp8.Fp8Matrix(codes, scale)
    dense = [_w(4096, 1024, g) for _ in range(2)]
    x = _x(4, 1024, g)
    want = [fp8.Fp8Matrix.from_dense(d).linear(x) for d in dense]
    y = []
    for i in range(20):
        assert sp._lib.sp_fp8_quantize_blocks(dense[i % 2].data_ptr(), 1024, 4096, 1024, codes.data_ptr(), 1024, scale.data_ptr(), sp._stream()) == 0
        y.append(w.linear(x))
    sp.check()
    assert all(torch.equal(v, want[i % 2]) for i, v in enumerate(y))


def test_workspace_is_shared_with_the_other_linears(sp, fp8):
    g = np.random.default_rng(0)
    wt, mask = synth.weight(600, 512, g), None
    mask = synth.magnitude_mask(wt, 60)
    h = sp.compress(gu.bf16_to_dev(wt), gu.u8_to_dev(mask))
    gt = _gen(8)
    for m in (3, 40, 300):
        x, w = _x(m, 512, gt), fp8.Fp8Matrix.from_dense(_w(600, 512, gt))
        ws = torch.zeros(max(h.workspace_size(m), w.workspace_size(m)), dtype=torch.uint8, device="cuda")
        a, b = h.linear(x), w.linear(x)
        for _ in range(3):
            assert torch.equal(h.linear(x, workspace=ws), a) and torch.equal(w.linear(x, workspace=ws), b)
    sp.check()


def test_linears_on_two_streams_at_once(sp, fp8):
    """Calls of every kind that overlap: each stream has its own workspace, and the rows' codes may be shared."""
    g = _gen(11)
    w = fp8.Fp8Matrix.from_dense(_w(2100, 1500, g))
    xs = [_x(m, 1500, g) for m in (1, 8, 40, 100, 600, 100, 3)]
    qs = [fp8.quantize_rows(x) for x in xs]
    want = [w.linear(x) for x in xs]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[] for _ in streams]
    for _ in range(5):
        for st, out in zip(streams, got):
            with torch.cuda.stream(st):
                out += [w.linear(x) for x in xs] + [w.linear(q) for q in qs]
    torch.cuda.synchronize()
    for out in got:
        for i, y in enumerate(out):
            assert torch.equal(y, want[i % 7]), i
    sp.check()


def test_tiles_that_are_shared_in_graphs_that_share_nothing(sp, fp8):
    """A batch whose tiles are shared by pairs, captured twice and replayed on two streams at once."""
    g = _gen(12)
    w = fp8.Fp8Matrix.from_dense(_w(1000, 9000, g))
    xs = [_x(150, 9000, g) for _ in range(2)]
    want = [w.linear(x) for x in xs]
    graphs, outs = [], []
    for x in xs:
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            outs.append(w.linear(x))
        graphs.append(gr)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(10):
        for st, gr in zip(streams, graphs):
            with torch.cuda.stream(st):
                gr.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    _check(outs[0], fp8.quantize_rows(xs[0]), w)
    sp.check()
