"""What Decoder.sample and Decoder.verify hand to the drawing of tokens (CPU: tensors that say they are on a GPU, a step that
only returns rows of logits, and calls that note what they get)."""
import types

import pytest
import torch

from paper_2405_03594_gb300 import decoder, serve
from tests.test_serve_devices import gpu

T, V, B = 5, 10, 2


@pytest.fixture
def calls(monkeypatch):
    """(a Decoder, the arguments of its calls of verify_drafts, which are checked as they are on a GPU)."""
    monkeypatch.setattr(serve, "_current_device", lambda: 0)
    monkeypatch.setattr(serve, "_stream", lambda *_: 0)
    monkeypatch.setattr(serve, "_verify", lambda *_: 0)
    monkeypatch.setattr(decoder, "token_probs", lambda logits, *_: gpu(torch.zeros(logits.shape, dtype=torch.float32)))
    seen = []

    def verify_drafts(*a):
        a = [gpu(x) if isinstance(x, torch.Tensor) else x for x in a]  # (new host tensors do not say where they are)
        seen.append(a)
        return serve.verify_drafts(*a)

    monkeypatch.setattr(decoder, "verify_drafts", verify_drafts)
    d = decoder.Decoder.__new__(decoder.Decoder)
    d.h = torch.zeros((8, 4), dtype=torch.bfloat16)
    d.head = types.SimpleNamespace(n=V)
    c = serve.KvCache(4, 2, 64, 16, data=torch.zeros(4 * 2 * 16 * 72, dtype=torch.uint8))
    d.batch = serve.Batch(c, 4, B, 8, 1)
    object.__setattr__(d.batch, "_gpu", 0)
    monkeypatch.setattr(serve.Batch, "retract", lambda *a, **k: None)
    d.step = lambda ids, *_: torch.zeros((ids.shape[0], V), dtype=torch.bfloat16)
    return d, seen


def _both(d, ids):
    new, w, u = gpu(torch.tensor([3, 2], dtype=torch.int32)), gpu(torch.zeros(B)), gpu(torch.zeros(T))
    d.sample(ids, new, 3, w)
    d.verify(ids, new, 3, gpu(torch.ones(B, dtype=torch.int32)), u, w)


def test_a_batch_with_longer_tables(calls):
    """A longer cu_q may take the place of a batch's own; the requests stay as many as they are."""
    d, seen = calls
    d.batch.__dict__["cu_q"] = gpu(torch.zeros(2 * B + 5, dtype=torch.int32))
    _both(d, gpu(torch.zeros(T, dtype=torch.int64)))
    assert [a[2].shape[0] for a in seen] == [B + 1, B + 1]


@pytest.mark.parametrize("dtype", [torch.int64, torch.int32])
def test_ids_at_any_stride(calls, dtype):
    """Ids that a step takes, such as a column of a table, are drawn behind as well."""
    d, seen = calls
    table = torch.arange(3 * T).view(T, 3).to(dtype)
    _both(d, gpu(table)[:, 1])
    for a in seen:
        assert a[1].tolist() == list(range(1, 3 * T, 3))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float64])
def test_under_another_default_type(calls, dtype):
    """PyTorch's default type is the caller's own; the random numbers that nothing reads are float32 all the same."""
    d, seen = calls
    ids, new, w = gpu(torch.zeros(T, dtype=torch.int64)), gpu(torch.tensor([3, 2], dtype=torch.int32)), gpu(torch.zeros(B))
    before = torch.get_default_dtype()
    torch.set_default_dtype(dtype)
    try:
        d.sample(ids, new, 3, w)
    finally:
        torch.set_default_dtype(before)
    assert seen[0][4].dtype == torch.float32 and seen[0][4].shape == (T,)
