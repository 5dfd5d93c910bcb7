"""The serving operators run together: a small compressed model prefills ragged prompts and decodes; the
queries, the attention and the rest of each layer, from the GPU's own inputs to each, in float64, with the
values that the caches hold.  (Without normalisation the activations grow, and a softmax of scores in the
hundreds magnifies what was rounded before it, so the stages are not chained in the comparison.)"""
import numpy as np
import pytest

from paper_2405_03594_gb300 import synth
from tests import gpu_util as gu
from tests import serve_ref as ref

pytestmark = pytest.mark.gpu

D_MODEL, HEADS, KV, DIM, FF, VOCAB, LAYERS = 256, 8, 2, 64, 320, 1000, 2
SHAPES = {"qkv": ((HEADS + 2 * KV) * DIM, D_MODEL), "o": (D_MODEL, HEADS * DIM), "gate_up": (2 * FF, D_MODEL),
          "down": (D_MODEL, FF)}


@pytest.fixture(scope="module")
def model():
    import torch

    from paper_2405_03594_gb300 import sp

    g = np.random.default_rng(0)

    def matrix(n, k, std):
        w = synth.weight(n, k, g, std=std)
        mask = synth.magnitude_mask(w, 60)
        return sp.compress(gu.bf16_to_dev(w), gu.u8_to_dev(mask)), synth.bf16_to_f32(w).astype(np.float64) * mask

    layers, dense = [], []
    for _ in range(LAYERS):
        pairs = {name: matrix(n, k, 1.2 / np.sqrt(0.4 * k)) for name, (n, k) in SHAPES.items()}
        layers.append({name: p[0] for name, p in pairs.items()})
        dense.append({name: p[1] for name, p in pairs.items()})
    head, dense_head = matrix(VOCAB, D_MODEL, 0.1)
    embed = torch.tensor(0.5 * g.standard_normal((VOCAB, D_MODEL)), device=gu.dev()).bfloat16()
    return layers, dense, head, dense_head, embed


def _decoder(model, requests=3, tokens=200, width=10, page_size=16):
    from paper_2405_03594_gb300.decoder import Decoder

    layers, _, head, _, embed = model
    return Decoder(layers, embed, head, HEADS, KV, 40, requests, tokens, width, page_size=page_size, positions=256)


def _i32(a):
    import torch

    return torch.tensor(a, dtype=torch.int32, device=gu.dev())


def _check(dec, model, record, new, logits):
    import torch

    _, dense, _, dense_head, embed = model
    lens, table = dec.batch.lens.tolist(), dec.batch.table.tolist()
    cs = dec.cos_sin.double().cpu().numpy()
    P = dec.batch.page_size
    pos = np.concatenate([np.arange(n - a, n) for n, a in zip(lens, new)]).astype(int)
    last = gu.bf16_from_dev(record[-1])

    def near(got, want):  # a few bf16 roundings (2^-9 each, of terms that add up like random ones)
        assert np.linalg.norm(got - want) <= 2.5e-2 * np.linalg.norm(want)

    for i, (w, cache, stage) in enumerate(zip(dense, dec.caches, record)):
        h, q, o = (gu.bf16_from_dev(t) for t in stage)
        x = (h @ w["qkv"].T).reshape(len(h), HEADS + 2 * KV, DIM)
        near(q, ref.rotate(x[:, :HEADS], cs[pos, :DIM // 2], cs[pos, DIM // 2:], False))
        out, at = [], 0
        for b, (n, a) in enumerate(zip(lens, new)):
            if a == 0:
                continue
            slots = torch.tensor([table[b][i // P] * P + i % P for i in range(n)], device=gu.dev())
            k, v = (t.double().cpu().numpy() for t in cache.read(slots))
            out.append(ref.attend(q[at:at + a], k, v, DIM ** -0.5))
            # what this step wrote: the keys rotated, the values as they are, to half a step of the 16 codes
            for got, want in ((k[n - a:], ref.rotate(x[:, HEADS:HEADS + KV], cs[pos, :DIM // 2], cs[pos, DIM // 2:], False)),
                              (v[n - a:], x[:, HEADS + KV:])):
                y = want[at:at + a]
                assert (np.abs(got - y) <= np.ptp(y, axis=-1, keepdims=True) * (0.5 / 15 + 2e-2)).all()
            at += a
        near(o, np.concatenate(out))
        h = h + o.reshape(len(h), -1) @ w["o"].T
        gu_ = h @ w["gate_up"].T
        near(gu.bf16_from_dev(record[i + 1][0]) if i + 1 < LAYERS else last, h + (gu_[:, 0::2] * gu_[:, 1::2]) @ w["down"].T)
    want = last @ dense_head.T
    gu.assert_close(gu.bf16_from_dev(logits), want)


def test_prefill_then_decode(model):
    import torch

    from paper_2405_03594_gb300 import sp

    dec = _decoder(model)
    g = torch.Generator().manual_seed(1)
    new = [70, 1, 33]
    ids = torch.randint(0, VOCAB, (sum(new),), generator=g).to(gu.dev())
    record = []
    logits = dec.step(ids, _i32(new), max(new), record=record)
    sp.check()
    assert dec.batch.status.item() == 0
    _check(dec, model, record, new, logits)
    for step in range(18):  # across page boundaries; the second request pauses, the third gets two tokens at once
        new = [1, step % 2, 2 if step == 3 else 1]
        ids = torch.randint(0, VOCAB, (sum(new),), generator=g).to(gu.dev())
        record = []
        logits = dec.step(ids, _i32(new), max(new), record=record)
        if step in (0, 3, 17):
            sp.check()
            _check(dec, model, record, new, logits)
    assert dec.batch.cached.tolist() == [70 + 18, 1 + 9, 33 + 19]
    before = dec.batch.free_count.item()
    dec.batch.plan(_i32([-1, 0, 0]), advance=True)  # the first request ends
    assert dec.batch.free_count.item() == before + -(-88 // 16) and dec.batch.cached.tolist() == [0, 10, 52]


def test_decode_in_a_graph_and_greedy_choice(model):
    """A captured decode step grows its requests at every replay, as the eager one does."""
    import torch

    from paper_2405_03594_gb300 import sp

    a, b = _decoder(model), _decoder(model)
    g = torch.Generator().manual_seed(2)
    new = [40, 7, 17]
    ids = torch.randint(0, VOCAB, (sum(new),), generator=g).to(gu.dev())
    la, lb = a.step(ids, _i32(new), 40).clone(), b.step(ids, _i32(new), 40).clone()
    assert torch.equal(la, lb)
    one, last = _i32([1, 1, 1]), torch.tensor([39, 46, 63], device=gu.dev())
    ia, ib = la[last].float().argmax(-1), lb[last].float().argmax(-1)
    b.step(ib, _i32([0, 0, 0]), 1)  # (per-device attributes are set outside the capture)
    torch.cuda.synchronize()
    graph, cell = torch.cuda.CUDAGraph(), ib.clone()
    with torch.cuda.graph(graph):
        nxt, lp, ent, tl, ti = b.greedy(cell, one, 1, top=4)
        cell.copy_(nxt)
    for _ in range(20):
        na, pa, ea, ta, ka = a.greedy(ia, one, 1, top=4)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(na, cell) and torch.equal(pa, lp) and torch.equal(ea, ent)
        assert torch.equal(ka, ti) and torch.equal(ta, tl) and torch.equal(a.logits[:3], b.logits[:3])
        x = a.logits[:3].double()
        assert torch.equal(x.gather(1, na[:, None])[:, 0], x.amax(-1))
        want = torch.log_softmax(x, -1).gather(1, ka)
        assert torch.allclose(ta.double(), want, atol=1e-5)
        ia = na
    assert a.batch.cached.tolist() == b.batch.cached.tolist() == [60, 27, 37]
    sp.check()


def test_a_step_that_does_not_fit_writes_nothing(model):
    import torch

    from paper_2405_03594_gb300 import sp

    dec = _decoder(model, width=2)
    ids = torch.zeros(40, dtype=torch.int64, device=gu.dev())
    dec.step(ids[:30], _i32([30, 0, 0]), 30)
    sp.check()
    kept = [c.data.clone() for c in dec.caches]
    dec.step(ids[:3], _i32([3, 0, 0]), 3)  # 33 tokens: more than two pages
    sp.check()
    assert dec.batch.status.item() == 2 and dec.batch.cached.tolist() == [30, 0, 0]
    for c, k in zip(dec.caches, kept):
        assert torch.equal(c.data, k)
