"""Rows quantised where there are many of them, four pairs of blocks to a warp: codes and scales are defined bit for bit and
equal those of the model, at row counts and lengths whose last group, pair and block are not full."""
import numpy as np
import pytest
import torch

from paper_2405_03594_gb300 import synth
from tests import drafts_ref as ref
from tests import gpu_util as gu

pytestmark = pytest.mark.gpu


def _rows(m, k, seed):
    g = np.random.default_rng(seed)
    x = g.standard_normal((m, k)) * np.exp(3 * g.standard_normal((m, 1)))
    x[g.random((m, k)) < 0.01] *= 50
    x[m // 2] = 0
    return synth.bf16_from_f32(x.astype(np.float32))


def _same(got, q, s):
    assert np.array_equal(got.scale.cpu().numpy(), s)
    assert np.array_equal(got.codes.double().cpu().numpy(), q)
    assert not got._codes[:, got.k:].any()


# row-pairs m * ceil(k / 256) from 16384 on, and four pairs or more of a row; the last three are below one of them
@pytest.mark.parametrize("m,k", [(4100, 1000), (3300, 1281), (4096, 769), (2731, 1537), (1171, 3329), (700, 6017), (373, 11008), (4095, 1024), (6000, 700)])
def test_many_rows_are_quantised_bit_for_bit(m, k):
    from paper_2405_03594_gb300 import fp8, sp

    bits = _rows(m, k, m + k)
    got = fp8.quantize_rows(gu.bf16_to_dev(bits))
    sp.check()
    _same(got, *ref.quantize(synth.bf16_to_f32(bits), 1))


@pytest.mark.parametrize("a", [1, 8])  # rows off 16 bytes, and on them
def test_many_rows_of_a_view(a):
    from paper_2405_03594_gb300 import fp8, sp

    m, k = 3300, 1270
    bits = _rows(m, 1288, a)
    got = fp8.quantize_rows(gu.bf16_to_dev(bits)[:, a:a + k])
    sp.check()
    _same(got, *ref.quantize(synth.bf16_to_f32(np.ascontiguousarray(bits[:, a:a + k])), 1))


def test_many_rows_with_numbers_that_are_not_finite():
    from paper_2405_03594_gb300 import fp8, sp

    m, k = 4100, 1000
    x = gu.bf16_to_dev(_rows(m, k, 7))
    clean = fp8.quantize_rows(x)
    x[5, 130], x[4099, 999], x[2000, 0] = float("nan"), float("inf"), float("-inf")
    got = fp8.quantize_rows(x)
    sp.check()
    hit = [(5, 1), (4099, 7), (2000, 0)]
    s = got.scale
    assert s[5, 1].isnan() and s[4099, 7] == torch.inf and s[2000, 0] == torch.inf
    other = torch.ones_like(s, dtype=torch.bool)
    for r, b in hit:
        other[r, b] = False
    assert torch.equal(s[other], clean.scale[other])
    each = other.repeat_interleave(128, 1)[:, :k]
    assert torch.equal(got.codes.view(torch.uint8)[each], clean.codes.view(torch.uint8)[each])


def test_nothing_behind_the_last_block_is_written():
    from paper_2405_03594_gb300 import fp8, sp

    m, k, stride, scale_stride = 4100, 900, 1280, 4160
    x = gu.bf16_to_dev(_rows(m, k, 9))
    want = fp8.quantize_rows(x)
    codes = torch.full((m + 1, stride), 0xaa, dtype=torch.uint8, device="cuda")
    scale = torch.full((9, scale_stride), 7.0, device="cuda")
    assert sp._lib.sp_fp8_quantize_rows(x.data_ptr(), k, m, k, codes.data_ptr(), stride, scale.data_ptr(), scale_stride, sp._stream()) == 0
    sp.check()
    assert torch.equal(codes[:m, :k], want.codes.view(torch.uint8)) and not codes[:m, k:1024].any()
    assert (codes[:m, 1024:] == 0xaa).all() and (codes[m] == 0xaa).all()
    assert torch.equal(scale[:8, :m].t(), want.scale) and (scale[:8, m:] == 7).all() and (scale[8] == 7).all()
