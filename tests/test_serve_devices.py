"""The serving calls' checks of where their tensors are: whatever hands an address to a kernel has to be on
the GPU of the call (CPU: tensors that say they are on a GPU stand in for those that are)."""
import pytest
import torch

from paper_2405_03594_gb300 import serve


class OnGpu(torch.Tensor):
    """A host tensor that says that it is on GPU 0; no call below gets as far as its address."""

    is_cuda = True

    def get_device(self):
        return 0


class Stream:
    cuda_stream = 0


def gpu(x):
    return x.as_subclass(OnGpu)


@pytest.fixture(autouse=True)
def _current(monkeypatch):
    if hasattr(serve, "_current_device"):
        monkeypatch.setattr(serve, "_current_device", lambda: 0)


def _cache(on_gpu):
    data = torch.zeros(4 * 2 * 16 * 72, dtype=torch.uint8)
    return serve.KvCache(4, 2, 64, 16, data=gpu(data) if on_gpu else data)


def _tensors():
    return dict(q=torch.zeros((3, 4, 64), dtype=torch.bfloat16), k=torch.zeros((3, 2, 64), dtype=torch.bfloat16),
                v=torch.zeros((3, 2, 64), dtype=torch.bfloat16), positions=torch.zeros(3, dtype=torch.int32),
                slots=torch.zeros(3, dtype=torch.int64), cos_sin=torch.zeros((4, 64)),
                q_weight=torch.zeros(64, dtype=torch.bfloat16), k_weight=torch.zeros(64, dtype=torch.bfloat16),
                out=torch.zeros((3, 4, 64), dtype=torch.bfloat16))


def _refused(call, what="GPU"):
    with pytest.raises(ValueError, match=what):
        call()


def test_a_cache_outside_the_calls_gpu_is_refused():
    c, t = _cache(False), {k: gpu(x) for k, x in _tensors().items()}
    _refused(lambda: c.append(**t, stream=Stream), "buffer")
    _refused(lambda: c.read(t["slots"], stream=Stream), "buffer")
    b = serve.Batch(c, 4, 1, 3, 1)
    ws = gpu(torch.zeros(1 << 25, dtype=torch.uint8))
    _refused(lambda: c.attend(t["q"], b, 3, out=t["out"], workspace=ws, stream=Stream), "buffer")
    _refused(lambda: _cache(True).attend(t["q"], b, 3, out=t["out"], workspace=ws, stream=Stream), "batch")
    _refused(lambda: b.plan(t["positions"][:1], stream=Stream), "batch")


@pytest.mark.parametrize("name", list(_tensors()))
def test_one_tensor_elsewhere_is_refused(name):
    t = {k: x if k == name else gpu(x) for k, x in _tensors().items()}
    _refused(lambda: _cache(True).append(**t, stream=Stream))


def test_tensors_of_another_gpu_than_the_current_one_are_refused(monkeypatch):
    monkeypatch.setattr(serve, "_current_device", lambda: 1)
    t = {k: gpu(x) for k, x in _tensors().items()}
    _refused(lambda: _cache(True).append(**t, stream=Stream))
    _refused(lambda: serve.token_logprobs(t["cos_sin"], t["slots"], stream=Stream))
    _refused(lambda: _cache(True).read(t["slots"], stream=Stream))


def test_ids_and_logits_on_two_devices_are_refused():
    t = _tensors()
    _refused(lambda: serve.token_logprobs(gpu(t["cos_sin"][:3]), t["slots"], stream=Stream))
    _refused(lambda: serve.token_logprobs(t["cos_sin"][:3], gpu(t["slots"]), stream=Stream))


def test_a_batchs_tables_keep_their_type_and_size():
    """A table that is exchanged for a smaller one, or one of other entries, would be read past its end."""
    b = serve.Batch(_cache(False), 4, 3, 5, 2)
    i32 = dict(dtype=torch.int32)
    good = dict(cached=torch.ones(3, **i32), table=torch.ones((3, 2), **i32), free=torch.ones(4, **i32),
                free_count=torch.ones(1, **i32), lens=torch.ones(3, **i32), next_count=torch.ones(1, **i32),
                cu_q=torch.ones(4, **i32), work=torch.ones(12, **i32), slots=torch.ones(5, dtype=torch.int64),
                positions=torch.ones(5, **i32), status=torch.ones(1, **i32))
    for name, x in good.items():
        setattr(b, name, x)
        assert getattr(b, name) is x
        wide = torch.ones((*x.shape[:-1], 2 * x.shape[-1]), dtype=x.dtype)
        for bad in (x[:0], x.float(), x.to(torch.int64 if x.dtype == torch.int32 else torch.int32), gpu(x), None,
                    *([wide[..., ::2]] if x.numel() > 1 else [])):
            with pytest.raises(ValueError, match=name):
                setattr(b, name, bad)
        assert getattr(b, name) is x
        if x.dim() == 1:
            setattr(b, name, wide)
    for name in ("heads", "kv_heads", "page_size", "pages", "requests", "tokens", "width"):
        with pytest.raises(AttributeError):
            setattr(b, name, 100)
    with pytest.raises(AttributeError):
        _cache(False).data = torch.zeros(5, dtype=torch.uint8)


def test_a_workspace_elsewhere_or_of_other_entries_is_refused():
    c = _cache(True)
    b, q = serve.Batch(_cache(False), 4, 1, 3, 1), gpu(_tensors()["q"])
    b.__dict__["_gpu"] = 0  # (a batch makes its tables where the buffer is)
    ws = torch.zeros(1 << 25, dtype=torch.uint8)
    for bad in (ws, gpu(ws)[::2], gpu(ws.view(torch.int32))):
        _refused(lambda: c.attend(q, b, 3, out=torch.empty_like(q), workspace=bad, stream=Stream), "workspace")


def test_a_cache_of_more_bytes_than_an_offset_holds_is_refused():
    """2^52 pages of 32 heads of 128: 136 * 2^64 bytes, which a 64-bit product takes for none."""
    import ctypes

    from paper_2405_03594_gb300 import sp

    b = ctypes.c_size_t()
    for pages, heads in ((1 << 52, 32), (1 << 62, 1), ((1 << 63) - 1, 1), (1 << 33, 1 << 30)):
        c = sp.SpKv4(1 << 20, pages, 128, heads, 128, 0)
        assert sp._lib.sp_kv4_bytes(c, ctypes.byref(b)) == 2, pages
        assert sp._lib.sp_kv4_read(c, 1 << 20, 1, 1 << 20, 1 << 20, None) == 2, pages
        with pytest.raises(sp.SpError):
            serve.KvCache(pages, heads, 128, 128, data=torch.zeros(0, dtype=torch.uint8))
    most = ((1 << 63) - 1) // (128 * 136)
    assert sp._lib.sp_kv4_bytes(sp.SpKv4(None, most, 128, 1, 128, 0), ctypes.byref(b)) == 0
    assert b.value == most * 128 * 136
    assert sp._lib.sp_kv4_bytes(sp.SpKv4(None, most + 1, 128, 1, 128, 0), ctypes.byref(b)) == 2
