"""The calls for drafted tokens and 8-bit linears: their checks of arguments, which return before any GPU work, and the
models that the GPU tests compare with, on hand-made values (CPU)."""
import ctypes
import math
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

from tests import drafts_ref as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 1 << 20  # an address that no call below gets to use


@pytest.fixture(scope="module")
def sp():
    from paper_2405_03594_gb300 import sp as _sp

    return _sp


def _set(c, **kw):
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def test_retract_refusals(sp):
    def args(**kw):
        a = sp.SpKvRetractArgs()
        for n in ("cached", "drop", "table", "free_pages", "free_count", "next_count", "lens", "status"):
            setattr(a, n, FAKE)
        return _set(_set(a, pages=4, requests=2, width=2, page_size=16), **kw)

    f = lambda a: sp._lib.sp_kv_retract(a, None)  # noqa: E731
    assert f(None) == 1
    for kw in (dict(requests=-1), dict(width=-1), dict(pages=-1), dict(page_size=24), dict(page_size=0), dict(reserved=1),
               dict(cached=None), dict(drop=None), dict(table=None), dict(free_count=None), dict(next_count=None),
               dict(lens=None), dict(status=None)):
        assert f(args(**kw)) == 1, kw
    assert f(args(pages=1 << 31)) == 2


def test_probs_refusals(sp):
    def call(logits=FAKE, dtype=0, stride=100, tokens=2, vocab=100, temperature=None, one=1.0, min_p=0.0, out=2 * FAKE, out_stride=100):
        return sp._lib.sp_token_probs(logits, dtype, stride, tokens, vocab, temperature, one, min_p, out, out_stride, None)

    for kw in (dict(dtype=2), dict(tokens=-1), dict(vocab=0), dict(stride=99), dict(out_stride=99), dict(min_p=-0.1),
               dict(min_p=1.1), dict(min_p=math.nan), dict(one=math.nan), dict(logits=None), dict(out=None),
               dict(out=FAKE), dict(out=FAKE + 396), dict(out=FAKE - 796), dict(dtype=1, out=FAKE + 796)):
        assert call(**kw) == 1, kw
    assert call(vocab=1 << 31, stride=1 << 31, out_stride=1 << 31) == 2
    for kw in (dict(logits=FAKE + 1), dict(logits=FAKE + 2, dtype=1), dict(out=FAKE + 2), dict(temperature=FAKE + 2)):
        assert call(**kw) == 3, kw
    assert call(tokens=0) == 0


def test_verify_refusals(sp):
    def args(**kw):
        a = sp.SpVerifyArgs()
        for n in ("probs", "ids", "cu_q", "drafts", "accept", "sample", "accepted", "rejected", "next"):
            setattr(a, n, FAKE)
        return _set(_set(a, stride=100, draft_stride=100, rows=3, vocab=100, requests=1, dtype=1, draft_dtype=1), **kw)

    f = lambda a: sp._lib.sp_verify_drafts(a, None)  # noqa: E731
    assert f(None) == 1
    for kw in (dict(requests=-1), dict(rows=-1), dict(vocab=0), dict(stride=99), dict(draft_probs=FAKE, draft_stride=99),
               dict(dtype=2), dict(draft_dtype=-1), dict(reserved=1), dict(probs=None), dict(ids=None), dict(cu_q=None),
               dict(drafts=None), dict(accept=None), dict(sample=None), dict(accepted=None), dict(rejected=None), dict(next=None)):
        assert f(args(**kw)) == 1, kw
    assert f(args(vocab=(1 << 22) + 1, stride=1 << 23)) == 2
    for kw in (dict(probs=FAKE + 2), dict(probs=FAKE + 1, dtype=0), dict(draft_probs=FAKE + 2)):
        assert f(args(**kw)) == 3, kw
    assert f(args(requests=0)) == 0


def test_quantize_refusals(sp):
    def rows(x=FAKE, xs=100, m=2, k=100, codes=FAKE, stride=112, scale=FAKE, ss=4):
        return sp._lib.sp_fp8_quantize_rows(x, xs, m, k, codes, stride, scale, ss, None)

    def blocks(w=FAKE, ws=100, n=2, k=100, codes=FAKE, stride=112, scale=FAKE):
        return sp._lib.sp_fp8_quantize_blocks(w, ws, n, k, codes, stride, scale, None)

    for kw in (dict(x=None), dict(xs=99), dict(m=-1), dict(k=0), dict(codes=None), dict(stride=96), dict(scale=None), dict(ss=1)):
        assert rows(**kw) == 1, kw
    for kw in (dict(stride=104), dict(ss=6), dict(m=(1 << 30) + 1, ss=1 << 31), dict(k=(1 << 30) + 1, xs=1 << 31, stride=1 << 31)):
        assert rows(**kw) == 2, kw
    for kw in (dict(x=FAKE + 1), dict(codes=FAKE + 8), dict(scale=FAKE + 8)):
        assert rows(**kw) == 3, kw
    assert rows(m=0) == 0
    for kw in (dict(w=None), dict(ws=99), dict(n=-1), dict(k=0), dict(codes=None), dict(stride=96), dict(scale=None)):
        assert blocks(**kw) == 1, kw
    for kw in (dict(stride=104), dict(n=(1 << 30) + 1)):
        assert blocks(**kw) == 2, kw
    for kw in (dict(w=FAKE + 1), dict(codes=FAKE + 8), dict(scale=FAKE + 2)):
        assert blocks(**kw) == 3, kw
    assert blocks(n=0) == 0


def test_linear_refusals(sp):
    def args(q=False, **kw):
        a = sp.SpFp8LinearArgs()
        for n in ("w", "w_scale", "y"):
            setattr(a, n, FAKE)
        _set(a, w_stride=112, y_stride=50, m=2, n=50, k=100)
        _set(a, xq=FAKE, x_scale=FAKE, xq_stride=112, x_scale_stride=4) if q else _set(a, x=FAKE, x_stride=100)
        return _set(a, **kw)

    f = lambda a, ws=FAKE: sp._lib.sp_fp8_linear(a, ws, 1 << 40, None)  # noqa: E731
    assert f(None) == 1
    for kw in (dict(m=-1), dict(n=0), dict(k=0), dict(w=None), dict(w_scale=None), dict(w_stride=96), dict(y=None),
               dict(y_stride=49), dict(x=None), dict(x_stride=99), dict(xq=FAKE, x_scale=FAKE)):
        assert f(args(**kw)) == 1, kw
    for kw in (dict(x_scale=None), dict(xq_stride=96), dict(x_scale_stride=1), dict(xq=None), dict(x=FAKE)):
        assert f(args(True, **kw)) == 1, kw
    for kw in (dict(w_stride=104), dict(m=(1 << 30) + 1)):
        assert f(args(**kw)) == 2, kw
    for kw in (dict(xq_stride=104), dict(x_scale_stride=6)):
        assert f(args(True, **kw)) == 2, kw
    for kw in (dict(w=FAKE + 8), dict(w_scale=FAKE + 2), dict(x=FAKE + 1), dict(y=FAKE + 1)):
        assert f(args(**kw)) == 3, kw
    for kw in (dict(xq=FAKE + 8), dict(x_scale=FAKE + 8)):
        assert f(args(True, **kw)) == 3, kw
    assert f(args(), FAKE + 8) == 3
    assert f(args(m=0)) == 0
    b = ctypes.c_size_t()
    g = sp._lib.sp_fp8_workspace_size
    assert g(1, 1, 1, None) == 1 and g(-1, 1, 1, ctypes.byref(b)) == 1 and g(1, 0, 1, ctypes.byref(b)) == 1
    assert g((1 << 30) + 1, 1, 1, ctypes.byref(b)) == 2


def test_struct_layouts(sp, tmp_path):
    """The binding's structs are the headers' (gcc, no GPU)."""
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("gcc not found")
    pairs = {"sp_kv_retract_args": sp.SpKvRetractArgs, "sp_verify_args": sp.SpVerifyArgs, "sp_fp8_linear_args": sp.SpFp8LinearArgs}
    lines = ['#include <stdio.h>', '#include "sp_serve.h"', '#include "sp_fp8.h"', "int main(void) {"]
    for c, t in pairs.items():
        lines.append(f'printf("{c} %zu\\n", sizeof({c}));')
        lines += [f'printf("{c}.{n} %zu\\n", offsetof({c}, {n}));' for n, _ in t._fields_]
    lines += ["return 0; }"]
    src = tmp_path / "l.c"
    src.write_text("\n".join(lines))
    subprocess.check_call([gcc, "-std=c11", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "l")])
    got = dict(x.split() for x in subprocess.check_output([str(tmp_path / "l")], text=True).splitlines())
    for c, t in pairs.items():
        assert int(got[c]) == ctypes.sizeof(t)
        for n, _ in t._fields_:
            assert int(got[f"{c}.{n}"]) == getattr(t, n).offset, (c, n)


class OnGpu(torch.Tensor):
    """A host tensor that says that it is on GPU 0; no call below gets as far as its address."""

    is_cuda = True

    def get_device(self):
        return 0


class Stream:
    cuda_stream = 0


def gpu(x):
    return x.as_subclass(OnGpu)


def _refused(call, what=None):
    with pytest.raises(ValueError, match=what):
        call()


def _verify_tensors():
    return dict(probs=torch.zeros((3, 10)), ids=torch.zeros(3, dtype=torch.int64), cu_q=torch.zeros(2, dtype=torch.int32),
                drafts=torch.zeros(1, dtype=torch.int32), accept=torch.zeros(3), sample=torch.zeros(1), draft_probs=torch.zeros((3, 10)))


@pytest.mark.parametrize("name", list(_verify_tensors()))
def test_one_tensor_elsewhere_or_of_another_kind_is_refused(monkeypatch, name):
    from paper_2405_03594_gb300 import serve

    monkeypatch.setattr(serve, "_current_device", lambda: 0)
    t = {k: gpu(x) for k, x in _verify_tensors().items()}
    for bad in (_verify_tensors()[name], t[name].to(torch.float16), gpu(torch.zeros((0, 3, 3)))):
        _refused(lambda: serve.verify_drafts(**{**t, name: bad}, stream=Stream))
    if name in ("ids", "drafts", "accept", "sample"):
        _refused(lambda: serve.verify_drafts(**{**t, name: t[name][:0]}, stream=Stream), name)
    if "probs" in name:
        _refused(lambda: serve.verify_drafts(**{**t, name: gpu(torch.zeros((10, 3)).t())}, stream=Stream), name)
    monkeypatch.setattr(serve, "_current_device", lambda: 1)
    _refused(lambda: serve.verify_drafts(**t, stream=Stream), "current")


def test_probabilities_and_tables_elsewhere_are_refused(monkeypatch):
    from paper_2405_03594_gb300 import serve

    monkeypatch.setattr(serve, "_current_device", lambda: 0)
    x, t, out = gpu(torch.zeros((3, 10))), gpu(torch.ones(3)), gpu(torch.zeros((3, 10)))
    for call in (lambda: serve.token_probs(torch.zeros((3, 10))), lambda: serve.token_probs(x, torch.ones(3), stream=Stream),
                 lambda: serve.token_probs(x, t[:2], stream=Stream), lambda: serve.token_probs(x, t.double(), stream=Stream),
                 lambda: serve.token_probs(x, t, out=torch.zeros((3, 10)), stream=Stream),
                 lambda: serve.token_probs(x, t, out=out[:2], stream=Stream),
                 lambda: serve.token_probs(x, t, out=out.bfloat16(), stream=Stream),
                 lambda: serve.token_probs(x.half(), t, stream=Stream), lambda: serve.token_probs(x[:, :0], t, stream=Stream)):
        _refused(call)
    c = serve.KvCache(4, 2, 64, 16, data=torch.zeros(4 * 2 * 16 * 72, dtype=torch.uint8))
    b = serve.Batch(c, 4, 2, 3, 1)
    drop = torch.zeros(2, dtype=torch.int32)
    _refused(lambda: b.retract(drop), "batch")
    b.__dict__["_gpu"] = 0
    _refused(lambda: b.retract(drop, stream=Stream), "drop")
    _refused(lambda: b.retract(gpu(drop[:1]), stream=Stream), "drop")
    _refused(lambda: b.retract(gpu(drop.long()), stream=Stream), "drop")


def test_eight_bit_tensors_elsewhere_or_of_another_kind_are_refused(monkeypatch):
    from paper_2405_03594_gb300 import fp8, serve

    monkeypatch.setattr(serve, "_current_device", lambda: 0)
    codes, scale = gpu(torch.zeros((130, 48), dtype=torch.uint8)), gpu(torch.zeros((2, 1)))
    for call in (lambda: fp8.Fp8Matrix(torch.zeros((130, 48), dtype=torch.uint8), scale),
                 lambda: fp8.Fp8Matrix(codes, torch.zeros((2, 1))), lambda: fp8.Fp8Matrix(codes, scale[:1]),
                 lambda: fp8.Fp8Matrix(codes.float(), scale), lambda: fp8.Fp8Matrix(codes, scale.double()),
                 lambda: fp8.Fp8Matrix(codes[0], scale), lambda: fp8.Fp8Matrix(codes.t(), gpu(torch.zeros((1, 2)))),
                 lambda: fp8.Fp8Matrix.from_dense(torch.zeros((4, 4), dtype=torch.bfloat16)),
                 lambda: fp8.quantize_rows(torch.zeros((4, 4), dtype=torch.bfloat16)),
                 lambda: fp8.quantize_rows(gpu(torch.zeros((4, 4))), stream=Stream),
                 lambda: fp8.quantize_rows(gpu(torch.zeros((4, 0), dtype=torch.bfloat16)), stream=Stream)):
        _refused(call)
    m = fp8.Fp8Matrix(codes, scale)
    m.__dict__["_ws"][3] = 256
    x, out, ws = gpu(torch.zeros((3, 48), dtype=torch.bfloat16)), gpu(torch.zeros((3, 130), dtype=torch.bfloat16)), gpu(torch.zeros(1 << 12, dtype=torch.uint8))
    good = dict(x=x, out=out, workspace=ws, stream=Stream)
    for bad in (dict(x=torch.zeros((3, 48), dtype=torch.bfloat16)), dict(x=x.float()), dict(x=x[:, :47]), dict(x=x[0]),
                dict(x=gpu(torch.zeros((48, 3), dtype=torch.bfloat16).t())), dict(out=out[:2]), dict(out=out[:, :129]), dict(out=out.float()),
                dict(out=torch.zeros((3, 130), dtype=torch.bfloat16)), dict(workspace=torch.zeros(1 << 12, dtype=torch.uint8)),
                dict(workspace=ws.float()), dict(workspace=ws[::2]),
                dict(x=fp8.Fp8Rows(torch.zeros((3, 48), dtype=torch.uint8), torch.zeros((1, 4)), 48)),
                dict(x=fp8.Fp8Rows(gpu(torch.zeros((3, 48), dtype=torch.uint8)), gpu(torch.zeros((1, 4))), 47))):
        _refused(lambda: m.linear(**{**good, **bad}))
    monkeypatch.setattr(serve, "_current_device", lambda: 1)
    _refused(lambda: m.linear(**good), "current")


def test_models_on_hand_made_values():
    v = ref.e4m3([0, 1, 17, 18, 19, 447, 464, 1e9, -3.3, 2.0 ** -10, 2.0 ** -9, 1.5 * 2.0 ** -9, np.nan])
    assert v[:-1].tolist() == [0, 1, 16, 18, 20, 448, 448, 448, -3.25, 0, 2.0 ** -9, 2.0 ** -8] and np.isnan(v[-1])
    t = torch.linspace(-460, 460, 200001).clamp(-448, 448)
    t = torch.cat([t, t * 1e-3, t * 2e-5])
    assert np.array_equal(ref.e4m3(t.numpy()), t.to(torch.float8_e4m3fn).double().numpy())
    assert np.array_equal(ref.E4M3, torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy(), equal_nan=True)
    q, s = ref.quantize(np.array([[448.0, -1, 0, 0.3]], np.float32), 1)
    assert s[0, 0] == 1 and q.tolist() == [[448, -1, 0, 0.3125]]
    q, s = ref.quantize(np.zeros((1, 3), np.float32), 128)
    assert not q.any() and s[0, 0] == 2.0 ** -100
    p = ref.probs(np.log(np.array([[1, 2, 1], [1, 4, 4], [1, 2, 1]], np.float32)), [1, 0, 0.5], 0)
    assert np.allclose(p, [[0.25, 0.5, 0.25], [0, 1, 0], [1 / 6, 4 / 6, 1 / 6]])
    assert np.allclose(ref.probs(np.log(np.array([[1, 2, 4]], np.float32)), [1], 0.4), [[0, 1 / 3, 2 / 3]])
    p = np.array([[0.5, 0.5, 0], [0.25, 0.25, 0.5], [0, 0, 1]], np.float32)
    q = np.array([[1, 0, 0], [0, 0.5, 0.5], [0, 0, 1]], np.float32)
    # u = 0.4 keeps token 0 (0.4 * 1 < 0.5), u = 0.5 refuses token 1 (0.5 * 0.5 < 0.25 is false): from (0.25, 0, 0)
    assert ref.verify(p, q, [9, 0, 1], [0, 3], [2], [0.4, 0.5, 0], [0.99]) == ([1], [1], [0])
    assert ref.verify(p, q, [9, 0, 1], [0, 3], [2], [0.4, 0.49, 0], [0.0]) == ([2], [0], [2])
    assert ref.verify(p, None, [9, 0, 1], [0, 3], [2], [0.5, 0, 0], [0.6]) == ([0], [2], [1])
    assert ref.verify(p, None, [9, 0, 1], [0, 0, 3], [0, 0], [0, 0, 0], [0.3, 0.3]) == ([0, 0], [0, 0], [-1, 2])
    assert ref.draw([1, 0, 3], 0.25) == 2 and ref.draw([1, 0, 3], 0.2499) == 0 and ref.draw([0, 0], 0.5) == -1
    assert ref.retract([33, 5, 16], [2, 0, 16], [[7, 8, 9], [1, 0, 0], [4, 0, 0]], [2], 16) == ([31, 5, 0], [2, 9, 4])
    assert ref.retract([3], [4], [[0]], [], 16) is None
