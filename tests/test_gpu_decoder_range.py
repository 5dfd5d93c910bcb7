"""The decoder at the ends of what it was made for: positions behind the given number, steps without tokens, and
more tokens than its buffers hold."""
import pytest

from tests import gpu_util as gu
from tests.test_gpu_decoder import HEADS, KV, VOCAB, _i32, model  # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu


def _decoder(model, positions, tokens=200, width=10):  # noqa: F811
    from paper_2405_03594_gb300.decoder import Decoder

    layers, _, head, _, embed = model
    return Decoder(layers, embed, head, HEADS, KV, 40, 3, tokens, width, page_size=16, positions=positions)


def test_positions_as_far_as_the_tables_reach(model):  # noqa: F811
    """A request may grow to its table's pages whatever `positions` says: its later tokens turn by their own
    angles, not by position 0's."""
    import torch

    from paper_2405_03594_gb300 import sp

    a, b = _decoder(model, 160), _decoder(model, 32)
    g = torch.Generator().manual_seed(5)
    for new in ([90, 20, 1], [70, 1, 33], [0, 1, 1]):
        ids = torch.randint(0, VOCAB, (sum(new),), generator=g).to(gu.dev())
        assert torch.equal(a.step(ids, _i32(new), max(new)), b.step(ids, _i32(new), max(new)))
        sp.check()


def test_a_step_without_tokens(model):  # noqa: F811
    import torch

    from paper_2405_03594_gb300 import sp

    dec = _decoder(model, 160)
    ids = torch.arange(30, device=gu.dev())
    dec.step(ids, _i32([20, 10, 0]), 20)
    logits = dec.step(ids[:0], _i32([-1, 0, 0]), 1)  # the first request ends
    sp.check()
    assert logits.shape == (0, VOCAB) and dec.batch.cached.tolist() == [0, 10, 0] and dec.batch.free_count.item() == 39
    nxt, logp, entropy, top_logp, top_ids = dec.greedy(ids[:0], _i32([0, 0, 0]), 1, top=3)
    assert nxt.shape == logp.shape == entropy.shape == (0,) and top_logp.shape == top_ids.shape == (0, 3)
    sp.check()


@pytest.mark.parametrize("what", ["count", "dtype", "dim", "device"])
def test_ids_that_the_step_cannot_take_change_nothing(model, what):  # noqa: F811
    import torch

    dec = _decoder(model, 160, tokens=20)
    ids = torch.zeros(12, dtype=torch.int64, device=gu.dev())
    dec.step(ids, _i32([12, 0, 0]), 12)
    bad = {"count": ids.repeat(2), "dtype": ids.float(), "dim": ids[None], "device": ids.cpu()}[what]
    held = dec.h.data_ptr(), dec.h.shape
    with pytest.raises(ValueError):
        dec.step(bad, _i32([0, 3, 0]), 3)
    assert dec.batch.cached.tolist() == [12, 0, 0] and (dec.h.data_ptr(), dec.h.shape) == held
