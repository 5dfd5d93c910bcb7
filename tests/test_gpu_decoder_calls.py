"""Calls of Decoder.sample and Decoder.verify that their documentation allows or refuses, beside the ordinary ones."""
import pytest

from tests import gpu_util as gu
from tests.test_gpu_decoder import HEADS, KV, VOCAB, _i32, model  # noqa: F401

pytestmark = pytest.mark.gpu


def _decoder(model, requests=3):  # noqa: F811
    from paper_2405_03594_gb300.decoder import Decoder

    layers, _, head, _, embed = model
    return Decoder(layers, embed, head, HEADS, KV, 40, requests, 200, 12, page_size=16, positions=256)


def _ids(n, seed=3):
    import torch

    return torch.randint(0, VOCAB, (n,), generator=torch.Generator().manual_seed(seed)).to(gu.dev())


def _tables(dec):
    b = dec.batch
    return [x.tolist() for x in (b.cached, b.free_count, b.free, b.table, b.cu_q, b.slots, b.status)]


def test_a_refused_call_can_be_made_again(model):  # noqa: F811
    """The tables are as they were, and the same call put right gives what a decoder gives that never saw the refused one."""
    import torch

    from paper_2405_03594_gb300 import sp

    a, b = _decoder(model), _decoder(model)
    ids, new = _ids(40), _i32([20, 13, 7])
    w, u, drafts = torch.full((3,), 0.4, device="cuda"), torch.full((40,), 0.01, device="cuda"), _i32([3, 0, 2])
    for d in (a, b):
        d.step(_ids(9, 4), _i32([4, 3, 2]), 4)
    before = _tables(a)
    for call in (lambda: a.sample(ids, new, 20, w[:2]), lambda: a.sample(ids, new, 20, w, w), lambda: a.sample(ids, new, 20, w, 1.0, 2.0),
                 lambda: a.verify(ids, new, 20, drafts[:2], u, w), lambda: a.verify(ids, new, 20, drafts, u[:39], w),
                 lambda: a.verify(ids, new, 20, drafts, u, w.double()), lambda: a.verify(ids, new, 20, drafts, u, w, torch.zeros((39, VOCAB), device="cuda")),
                 lambda: a.verify(ids, new, 20, drafts, u, w, None, float("nan")), lambda: a.verify(ids.view(2, 20), new, 20, drafts, u, w)):
        with pytest.raises((ValueError, sp.SpError)):
            call()
        assert _tables(a) == before
    q = torch.softmax(torch.randn((40, VOCAB), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda"), -1)
    got, want = (d.verify(ids, new, 20, drafts, u, w, q, 0.7) for d in (a, b))
    sp.check()
    assert all(torch.equal(x, y) for x, y in zip(got, want)) and _tables(a) == _tables(b)


def test_a_temperature_for_each_request(model):  # noqa: F811
    """Spread over the rows as the documentation says: each request's token is the one that it alone would get."""
    import torch

    from paper_2405_03594_gb300 import serve, sp

    dec = _decoder(model)
    each, new, w = torch.tensor([0.0, 0.5, 1.5], device="cuda"), _i32([2, -1, 1]), torch.full((3,), 0.7, device="cuda")
    rows = torch.repeat_interleave(each, new.clamp(min=0), output_size=3)
    nxt, p = dec.sample(_ids(3), new, 2, w, rows)
    sp.check()
    for r, t in enumerate((0.0, 0.0, 1.5)):
        assert torch.equal(p[r:r + 1], serve.token_probs(dec.logits[r:r + 1], t))
    assert nxt[0] == dec.logits[1].float().argmax() and nxt[1] == -1 and 0 <= nxt[2] < VOCAB


def test_ids_at_any_stride_longer_tables_and_another_default_type(model):  # noqa: F811
    import torch

    from paper_2405_03594_gb300 import sp

    a, b = _decoder(model), _decoder(model)
    b.batch.cu_q = torch.zeros(20, dtype=torch.int32, device="cuda")
    b.batch.cached = torch.zeros(9, dtype=torch.int32, device="cuda")
    ids, new = _ids(40), _i32([20, 13, 7])
    w, u = torch.full((3,), 0.4, device="cuda"), torch.full((40,), 0.002, device="cuda")
    column = torch.stack([ids, 0 * ids, ids], 1)[:, 2]
    assert column.stride(0) == 3
    for call in (lambda d, i: d.sample(i, new, 20, w, 0.8)[0], lambda d, i: torch.stack([x.long() for x in d.verify(i, new, 20, _i32([4, 2, 6]), u, w, None, 0.8)])):
        want = call(a, ids)
        torch.set_default_dtype(torch.bfloat16)
        try:
            got = call(b, column)
        finally:
            torch.set_default_dtype(torch.float32)
        assert torch.equal(got, want)
    sp.check()
    assert a.batch.cached.tolist() == b.batch.cached.tolist()[:3]
