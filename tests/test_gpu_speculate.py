"""The operators for drafted tokens run together, as they are used: a small dense model in 8 bits drafts, a compressed
model verifies, refused tokens leave the cache again, and the next round goes on behind the kept ones."""
import numpy as np
import pytest

from paper_2405_03594_gb300 import synth
from tests import drafts_ref as ref
from tests import gpu_util as gu
from tests.test_gpu_decoder import DIM, D_MODEL, HEADS, KV, SHAPES, VOCAB, _i32, model  # noqa: F401

pytestmark = pytest.mark.gpu


def _target(model, head=None, width=12, pages=40):  # noqa: F811
    from paper_2405_03594_gb300.decoder import Decoder

    layers, _, h, _, embed = model
    return Decoder(layers, embed, head or h, HEADS, KV, pages, 3, 200, width, page_size=16, positions=256)


def _draft(model):  # noqa: F811
    """One dense layer and a dense vocabulary, in 8 bits."""
    import torch

    from paper_2405_03594_gb300 import fp8
    from paper_2405_03594_gb300.decoder import Decoder

    g = torch.Generator(device="cuda").manual_seed(5)
    layer = {n: fp8.Fp8Matrix.from_dense((torch.randn(s, generator=g, device="cuda") * s[1] ** -0.5).bfloat16()) for n, s in SHAPES.items()}
    head = fp8.Fp8Matrix.from_dense((0.1 * torch.randn((VOCAB, D_MODEL), generator=g, device="cuda")).bfloat16())
    return Decoder([layer], model[4], head, HEADS, KV, 40, 3, 200, 12, page_size=16, positions=256)


def test_a_decoder_of_dense_layers_in_eight_bits(model):  # noqa: F811
    """Its logits from the hidden rows before them, in 64 bits, with the weights that the codes stand for; what
    quantising the rows and rounding adds is a few e4m3 steps, 2^-4 of a value, over sums of 256 random ones."""
    import torch

    from paper_2405_03594_gb300 import sp

    dec = _draft(model)
    ids = torch.randint(0, VOCAB, (75,), generator=torch.Generator().manual_seed(3)).to(gu.dev())
    record = []
    logits = dec.step(ids, _i32([70, 1, 4]), 70, record=record)
    sp.check()
    h = record[-1].double()
    want = h @ dec.head.dense().double().T
    got = logits.double()
    assert torch.isfinite(got).all() and (got - want).norm() <= 2.0 ** -4 * want.norm()
    q = record[0][0].double() @ dec.layers[0]["qkv"].dense().double().T
    x = q.view(75, HEADS + 2 * KV, DIM)
    k, v = dec.caches[0].read(dec.batch.slots[:75])
    spread = x[:, HEADS + KV:].amax(-1, keepdim=True) - x[:, HEADS + KV:].amin(-1, keepdim=True)
    assert ((v.double() - x[:, HEADS + KV:]).abs() <= spread * (0.5 / 15 + 2.0 ** -3)).all()


@pytest.mark.parametrize("temperature", [0.0, 0.8])
@pytest.mark.parametrize("certain", [False, True])
def test_rounds_of_drafts(model, temperature, certain):  # noqa: F811
    import torch

    from paper_2405_03594_gb300 import sp

    target, draft = _target(model), _draft(model)
    rng, g = np.random.default_rng(0), torch.Generator(device="cuda").manual_seed(1)
    prompts = [rng.integers(0, VOCAB, n).tolist() for n in (37, 1, 16)]
    tokens = [list(p) for p in prompts]  # what each request has, the last one not yet in any cache
    behind = [0, 0, 0]                   # of those, in the target's cache
    drafted = [0, 0, 0]                  # and in the draft's

    def rand(n):
        return torch.rand(n, generator=g, device="cuda")

    for step in range(12):
        # the draft catches up with the target and draws up to three tokens, request by request of its own
        counts = [3, step % 3, 2]
        ids = [t[n:] for t, n in zip(tokens, drafted)]
        rows = [[] for _ in tokens]
        news = [[] for _ in tokens]
        for k in range(max(counts)):
            give = [i if k < c else [] for i, c in zip(ids, counts)]
            flat = torch.tensor(sum(give, []), dtype=torch.int64, device=gu.dev())
            nxt, probs = draft.sample(flat, _i32([len(x) for x in give]), max(len(x) for x in give), rand(3), 0.9)
            cu = draft.batch.cu_q.tolist()
            for b in range(3):
                if k < counts[b]:
                    drafted[b] += len(ids[b])
                    rows[b].append(probs[cu[b + 1] - 1].clone())
                    news[b].append(nxt[b].item())
                    assert 0 <= news[b][-1] < VOCAB
                    ids[b] = [news[b][-1]]
        # the target looks at what it has not seen and at the drafts
        give = [t[n:] + d for t, n, d in zip(tokens, behind, news)]
        flat = torch.tensor(sum(give, []), dtype=torch.int64, device=gu.dev())
        t = flat.shape[0]
        q = None
        if not certain:
            q = torch.zeros((t, VOCAB), device="cuda")
            at = 0
            for b in range(3):
                at += len(give[b])
                for j, r in enumerate(rows[b]):
                    q[at - 1 - counts[b] + j] = r
        accept, sample = rand(t), rand(3)
        free = target.batch.free_count.item()
        a, r, nxt = target.verify(flat, _i32([len(x) for x in give]), max(len(x) for x in give), _i32(counts), accept, sample, q, temperature)
        sp.check()
        cu = np.cumsum([0] + [len(x) for x in give]).tolist()
        # the same decisions from the GPU's own probabilities
        from paper_2405_03594_gb300 import serve

        p = serve.token_probs(target.logits[:t], temperature).cpu().numpy()
        want = ref.verify(p, None if q is None else q.cpu().numpy(), flat.tolist(), cu, counts, accept.cpu().numpy(), sample.cpu().numpy())
        assert [a.tolist(), r.tolist(), nxt.tolist()] == [list(map(int, w)) for w in want]
        back = []
        for b in range(3):
            kept = a[b].item()
            behind[b] += len(give[b]) - counts[b] + kept
            tokens[b] += news[b][:kept] + [nxt[b].item()]
            assert behind[b] == len(tokens[b]) - 1
            # the draft forgets what was refused; a draft that was never fed back was not in its cache
            over = max(0, drafted[b] - behind[b])
            back.append(over)
            drafted[b] -= over
        assert target.batch.cached.tolist() == behind
        held = sum(-(-n // 16) for n in behind)
        assert target.batch.free_count.item() == 40 - held and free >= 0
        pages = [x for b in range(3) for x in target.batch.table[b, :-(-behind[b] // 16)].tolist()] + target.batch.free[:40 - held].tolist()
        assert sorted(pages) == list(range(40))
        draft.batch.retract(_i32(back), advance=True)
        assert draft.batch.cached.tolist() == drafted and draft.batch.status.item() == 0
    sp.check()
    assert all(len(t) > len(p) + 11 for t, p in zip(tokens, prompts))
    # The first layer's cache holds what a decoder that never saw a refused token holds.  (Further on the model, which has no
    # norms, magnifies roundings.)  The rows before the 4-bit codes come from other kernels, of other batch sizes: two
    # roundings to bf16 of nearly one sum differ by a unit, 2^-7 of a value, and a rotated pair by 2^-6 of the largest; a code then
    # stands for a value within half a step of its row, so that two differ by a step, 1/15 of the spread, more.
    fresh = _target(model)
    flat = torch.tensor(sum((t[:-1] for t in tokens), []), dtype=torch.int64, device=gu.dev())
    assert fresh.step(flat, _i32(behind), max(behind)).shape[0] == sum(behind)
    for b in range(3):
        i = torch.arange(behind[b], device="cuda")
        rows = [d.caches[0].read(d.batch.table[b].long()[i // 16] * 16 + i % 16) for d in (target, fresh)]
        for x, y in zip(*rows):
            x, y = x.double(), y.double()
            spread = y.amax(-1, keepdim=True) - y.amin(-1, keepdim=True)
            assert ((x - y).abs() <= spread * (1.02 / 15) + 2.0 ** -6 * y.abs().amax(-1, keepdim=True)).all()
    sp.check()


def test_drafts_of_the_model_itself_are_kept(model):  # noqa: F811
    """At temperature 0, drafts that are the target's own best tokens, and one that is not."""
    import torch

    from paper_2405_03594_gb300 import sp

    dec = _target(model)
    g = torch.Generator().manual_seed(7)
    ids = torch.randint(0, VOCAB, (30,), generator=g).to(gu.dev())
    nxt, _ = dec.sample(ids, _i32([30, 0, 0]), 30, torch.zeros(3, device="cuda"), 0.0)
    assert nxt.tolist()[1:] == [-1, -1] and nxt[0] == dec.logits[29].float().argmax()
    before = dec.batch.cached.tolist()
    wrong = torch.tensor([nxt[0].item(), 5, 6, 7], device=gu.dev())
    probe = dec.verify(wrong, _i32([4, 0, 0]), 4, _i32([3, 0, 0]), torch.zeros(4, device="cuda"), torch.zeros(3, device="cuda"), None, 0.0)
    best = dec.logits[:4].float().argmax(-1).tolist()
    a = next((i for i in range(3) if best[i] != [5, 6, 7][i]), 3)
    assert [x.tolist()[0] for x in probe] == [a, 3 - a, best[a]]
    assert dec.batch.cached.tolist() == [before[0] + 1 + a, 0, 0]
    sp.check()


def test_a_round_in_a_graph(model):  # noqa: F811
    """A captured verification, replayed: it goes on behind what each replay kept, as the eager calls do."""
    import torch

    from paper_2405_03594_gb300 import sp

    a, b = _target(model), _target(model)
    g = torch.Generator(device="cuda").manual_seed(2)
    ids = torch.randint(0, VOCAB, (60,), generator=g, device="cuda")
    for d in (a, b):
        d.step(ids[:50], _i32([20, 13, 17]), 20)
    new, drafts = _i32([4, 2, 3]), _i32([3, 1, 2])
    cell, u, w = ids[50:59].clone(), torch.zeros(9, device="cuda"), torch.zeros(3, device="cuda")
    b.verify(cell[:0], _i32([0, 0, 0]), 1, _i32([0, 0, 0]), u[:0], w, None, 0.7)  # (per-device attributes are set outside the capture)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = b.verify(cell, new, 4, drafts, u, w, None, 0.7)
    for _ in range(8):
        cell.copy_(torch.randint(0, VOCAB, (9,), generator=g, device="cuda"))
        u.copy_(0.002 * torch.rand(9, generator=g, device="cuda"))  # (random drafts: a few are kept all the same)
        w.copy_(torch.rand(3, generator=g, device="cuda"))
        want = a.verify(cell, new, 4, drafts, u, w, None, 0.7)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want)) and a.batch.cached.tolist() == b.batch.cached.tolist()
    sp.check()


def test_a_step_that_does_not_fit_keeps_its_status(model):  # noqa: F811
    import torch

    from paper_2405_03594_gb300 import sp

    dec = _target(model, width=2)
    ids = torch.zeros(40, dtype=torch.int64, device=gu.dev())
    u, w = torch.zeros(40, device="cuda"), torch.zeros(3, device="cuda")
    dec.step(ids[:30], _i32([30, 0, 0]), 30)
    a, r, nxt = dec.verify(ids[:3], _i32([3, 0, 0]), 3, _i32([2, 0, 0]), u[:3], w)  # 33 tokens: more than two pages
    sp.check()
    assert dec.batch.status.item() == 2 and dec.batch.cached.tolist() == [30, 0, 0]
    assert (a.tolist(), r.tolist(), nxt.tolist()) == ([0] * 3, [0] * 3, [-1] * 3)
