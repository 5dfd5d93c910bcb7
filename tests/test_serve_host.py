"""The serving calls' checks of arguments, which return before any GPU work, and the models that the
GPU tests compare with, on hand-made values (CPU)."""
import ctypes
import math
import os
import shutil
import subprocess

import numpy as np
import pytest

from tests import serve_ref as ref

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


def _cache(sp, **kw):
    return _set(sp.SpKv4(FAKE, 4, 16, 2, 64, 0), **kw)


def test_cache_bytes_and_refusals(sp):
    b = ctypes.c_size_t()
    f = sp._lib.sp_kv4_bytes
    assert f(_cache(sp), ctypes.byref(b)) == 0 and b.value == 4 * 2 * 16 * 72
    big = _cache(sp, pages=1 << 20, page_size=128, kv_heads=32, head_dim=128)
    assert f(big, ctypes.byref(b)) == 0 and b.value == (1 << 20) * 128 * 32 * 136
    assert f(None, ctypes.byref(b)) == 1 and f(_cache(sp), None) == 1
    for kw in (dict(pages=0), dict(kv_heads=0), dict(pages=-1), dict(reserved=1)):
        assert f(_cache(sp, **kw), ctypes.byref(b)) == 1, kw
    for kw in (dict(page_size=24), dict(page_size=0), dict(page_size=256), dict(head_dim=96)):
        assert f(_cache(sp, **kw), ctypes.byref(b)) == 2, kw


def test_plan_refusals(sp):
    def args(**kw):
        a = sp.SpKvPlanArgs()
        for n in ("cached", "new_tokens", "table", "free_pages", "free_count", "next_count", "lens", "cu_q", "work",
                  "slots", "positions", "status"):
            setattr(a, n, FAKE)
        return _set(_set(a, max_tokens=4, pages=4, requests=2, width=2, page_size=16, group=1), **kw)

    for kw in (dict(requests=-1), dict(width=-1), dict(max_tokens=-1), dict(pages=-1), dict(page_size=24),
               dict(page_size=0), dict(group=0), dict(group=65), dict(cu_q=None), dict(work=None), dict(status=None),
               dict(cached=None), dict(new_tokens=None), dict(table=None), dict(lens=None), dict(slots=None),
               dict(positions=None), dict(free_count=None), dict(next_count=None)):
        assert sp._lib.sp_kv_plan(args(**kw), None) == 1, kw
    for kw in (dict(max_tokens=1 << 31), dict(pages=1 << 31)):
        assert sp._lib.sp_kv_plan(args(**kw), None) == 2, kw
    assert sp._lib.sp_kv_plan(None, None) == 1


def test_rope_refusals(sp):
    c = _cache(sp)

    def args(cache=True, **kw):
        a = sp.SpRopeArgs()
        for n in ("q", "k", "q_out", "positions", "cos_sin"):
            setattr(a, n, FAKE)
        _set(a, q_stride=256, k_stride=128, rows=8, eps=1e-5, tokens=2, heads=4, kv_heads=2, head_dim=64, rot=64)
        if cache:
            _set(a, cache=ctypes.pointer(c), slots=FAKE, v=FAKE, v_stride=128)
        else:
            a.k_out = FAKE
        return _set(a, **kw)

    f = sp._lib.sp_qk_norm_rope
    assert f(None, None) == 1
    for kw in (dict(tokens=-1), dict(heads=0), dict(kv_heads=0), dict(rows=0), dict(rot=-16), dict(rot=80),
               dict(pairs=2), dict(slots=None), dict(v=None), dict(k_out=FAKE), dict(kv_heads=1), dict(q=None),
               dict(k=None), dict(q_out=None), dict(positions=None), dict(cos_sin=None), dict(q_stride=248),
               dict(k_stride=64), dict(v_stride=64), dict(head_dim=128, rot=64, q_stride=512, k_stride=256)):
        assert f(args(**kw), None) == 1, kw
    assert f(args(cache=False, k_out=None), None) == 1
    for kw in (dict(rot=24), dict(head_dim=96), dict(q_stride=260), dict(v_stride=132)):
        assert f(args(**kw), None) == 2, kw
    for n in ("q", "k", "v", "q_out", "cos_sin", "q_weight", "k_weight"):
        assert f(args(**{n: FAKE + 8}), None) == 3, n
    assert f(args(tokens=0), None) == 0
    bad = _cache(sp, page_size=48)
    assert f(_set(args(), cache=ctypes.pointer(bad)), None) == 2


def test_read_and_attend_refusals(sp):
    f = sp._lib.sp_kv4_read
    assert f(None, FAKE, 1, FAKE, FAKE, None) == 1
    assert f(_cache(sp, data=None), FAKE, 1, FAKE, FAKE, None) == 1
    assert f(_cache(sp, head_dim=32), FAKE, 1, FAKE, FAKE, None) == 2
    assert f(_cache(sp, data=FAKE + 4), FAKE, 1, FAKE, FAKE, None) == 3
    assert f(_cache(sp), FAKE, -1, FAKE, FAKE, None) == 1
    assert f(_cache(sp), None, 1, FAKE, FAKE, None) == 1
    assert f(_cache(sp), FAKE, 1, FAKE + 2, FAKE, None) == 3
    assert f(_cache(sp), FAKE, 0, FAKE, FAKE, None) == 0
    c = _cache(sp)

    def args(**kw):
        a = sp.SpAttendArgs()
        for n in ("q", "out", "table", "lens", "cu_q", "work"):
            setattr(a, n, FAKE)
        _set(a, q_stride=256, out_stride=256, cache=ctypes.pointer(c), tokens=2, requests=1, width=2, heads=4, max_new=2,
             scale=0.1)
        return _set(a, **kw)

    f = lambda a: sp._lib.sp_kv4_attend(a, FAKE, 1 << 30, None)  # noqa: E731
    assert f(None) == 1
    for kw in (dict(cache=None), dict(requests=-1), dict(width=-1), dict(tokens=-1), dict(max_new=-1),
               dict(scale=math.nan), dict(scale=math.inf), dict(heads=3), dict(heads=1), dict(reserved=1), dict(q=None),
               dict(out=None), dict(table=None), dict(lens=None), dict(cu_q=None), dict(work=None), dict(q_stride=128),
               dict(out_stride=128)):
        assert f(args(**kw)) == 1, kw
    for kw in (dict(heads=130, q_stride=130 * 64, out_stride=130 * 64), dict(q_stride=260), dict(out_stride=260)):
        assert f(args(**kw)) == 2, kw
    for n in ("q", "out"):
        assert f(args(**{n: FAKE + 8})) == 3, n
    assert sp._lib.sp_kv4_attend(args(), FAKE + 8, 1 << 30, None) == 3
    for kw in (dict(requests=0), dict(tokens=0), dict(max_new=0)):
        assert f(args(**kw)) == 0, kw
    b = ctypes.c_size_t()
    assert sp._lib.sp_kv4_attend_workspace_size(64, None) == 1
    assert sp._lib.sp_kv4_attend_workspace_size(80, ctypes.byref(b)) == 2


def test_logprobs_refusals(sp):
    def call(logits=FAKE, dtype=0, stride=100, tokens=2, vocab=100, ids=FAKE, top=0, lp=FAKE, en=FAKE, tl=FAKE, ti=FAKE):
        return sp._lib.sp_token_logprobs(logits, dtype, stride, tokens, vocab, ids, top, lp, en, tl, ti, None)

    for kw in (dict(dtype=2), dict(tokens=-1), dict(vocab=0), dict(stride=99), dict(top=-1), dict(top=65),
               dict(vocab=3, top=4), dict(logits=None), dict(ids=None), dict(lp=None), dict(en=None),
               dict(top=1, tl=None), dict(top=1, ti=None)):
        assert call(**kw) == 1, kw
    assert call(vocab=1 << 31, stride=1 << 31) == 2
    assert call(logits=FAKE + 1) == 3 and call(logits=FAKE + 2, dtype=1) == 3
    assert call(tokens=0) == 0


def test_tensors_outside_a_gpu_are_refused(sp):
    import torch

    from paper_2405_03594_gb300 import serve

    data = torch.zeros(4 * 2 * 16 * 72, dtype=torch.uint8)
    c = serve.KvCache(4, 2, 64, 16, data=data)
    q = torch.zeros((3, 4, 64), dtype=torch.bfloat16)
    pos, slots, cs = torch.zeros(3, dtype=torch.int32), torch.zeros(3, dtype=torch.int64), torch.zeros((4, 64))
    b = serve.Batch(c, 4, 1, 3, 1)
    for call in (lambda: c.append(q, q[:, :2], q[:, :2], pos, slots, cs), lambda: c.read(slots), lambda: c.attend(q, b, 3),
                 lambda: serve.qk_norm_rope(q, q[:, :2], pos, cs), lambda: b.plan(pos[:1]),
                 lambda: serve.token_logprobs(cs, slots)):
        with pytest.raises(ValueError, match="GPU"):
            call()


def test_struct_layouts(sp, tmp_path):
    """The binding's structs are the header's (gcc, no GPU)."""
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("gcc not found")
    pairs = {"sp_kv4": sp.SpKv4, "sp_kv_plan_args": sp.SpKvPlanArgs, "sp_rope_args": sp.SpRopeArgs,
             "sp_attend_args": sp.SpAttendArgs}
    lines = ['#include <stdio.h>', '#include "sp_serve.h"', "int main(void) {"]
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


def test_models_on_hand_made_values():
    n, s, m = ref.quantize(np.arange(16, dtype=np.float32)[None] * 2 - 3)
    assert n.tolist() == [list(range(16))] and s[0] == 2 and m[0] == -3
    assert np.array_equal(ref.values(n, s, m)[0], np.arange(16) * 2.0 - 3)
    n, s, m = ref.quantize(np.full((1, 16), 5, np.float32))
    assert not n.any() and s[0] == 0 and m[0] == 5
    n, s, m = ref.quantize(np.array([[1, np.inf, 2, 3]], np.float32))
    assert not n.any() and s[0] == 0 and np.isnan(m[0])
    x = np.arange(8, dtype=np.float32).reshape(1, 1, 8)
    c, s = np.zeros((1, 2), np.float32), np.ones((1, 2), np.float32)  # a quarter turn
    assert ref.rotate(x, c, s, False)[0, 0].tolist() == [-2, -3, 0, 1, 4, 5, 6, 7]
    assert ref.rotate(x, c, s, True)[0, 0].tolist() == [-1, 0, -3, 2, 4, 5, 6, 7]
    y = ref.norm(np.array([[3, 4, 0, 0]], np.float32), np.ones(4, np.float32), 0.0)
    assert np.allclose(y, [[1.2, 1.6, 0, 0]])
    k = np.zeros((3, 1, 2))
    v = np.arange(6.0).reshape(3, 1, 2)
    o = ref.attend(np.ones((2, 2, 2)), k, v, 1.0)  # equal scores: means of what is seen
    assert np.allclose(o[0, 0], [1, 2]) and np.allclose(o[1, 1], [2, 3])
    assert not ref.attend(np.ones((2, 1, 2)), k[:1], v[:1], 1.0)[0].any()  # sees nothing
    lp, en, tl, ti = ref.logprobs(np.log(np.array([[1.0, 4, 4, 1]])), [1], 3)
    assert np.allclose(lp, math.log(0.4)) and ti.tolist() == [[1, 2, 0]]
    assert np.allclose(en, -2 * (0.4 * math.log(0.4) + 0.1 * math.log(0.1)))
    t = ref.Tables([3, 4, 0], [[7, -1], [5, -1], [-1, -1]], [1, 2, 3], 4, 8)
    lens, cu, slots, pos, table, free, status = t.step([2, -1, 1])
    assert (lens, cu, status) == ([5, 0, 1], [0, 2, 2, 3], 0)
    assert table == [[7, 5], [5, -1], [3, -1]] and free == [1, 2]
    assert slots[:4] == [31, 20, 12, -1] and pos[:4] == [3, 4, 0, 0]
    assert t.step([100, 0, 0])[6] == 1 | 2 | 4
