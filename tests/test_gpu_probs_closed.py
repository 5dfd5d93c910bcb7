"""Rows of logits in which nothing is open (every entry -inf), at any temperature: they are NaN, as include/sp_serve.h says,
and nothing is drawn from them."""
import numpy as np
import pytest
import torch

from tests import drafts_ref as ref

TEMPERATURES = (0.0, -1.0, -np.inf, 1.0, np.inf)


def test_the_model_gives_nan_for_rows_without_an_open_entry():
    for v in (1, 5):
        got = ref.probs(np.full((len(TEMPERATURES), v), -np.inf, np.float32), TEMPERATURES, 0.0)
        assert np.isnan(got).all()
    # one open entry, or one of +inf, is the best one all the same
    x = np.full((2, 3), -np.inf, np.float32)
    x[0, 1], x[1, 2] = -3e38, np.inf
    assert ref.probs(x, [0, 0], 0.0).tolist() == [[0, 1, 0], [0, 0, 1]]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("v", [1, 2, 9, 801, 32000, 131071])  # (the longest rows have several CTAs)
@pytest.mark.parametrize("min_p", [0.0, 0.5])
def test_rows_without_an_open_entry_are_nan(dtype, v, min_p):
    from paper_2405_03594_gb300 import serve, sp

    t = len(TEMPERATURES)
    x = torch.full((2 * t, v), -torch.inf, dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda")
    x[t:, v - 1] = -2.0  # the rows behind have one open entry
    got = serve.token_probs(x, torch.tensor(2 * TEMPERATURES, device="cuda"), min_p=min_p)
    one = [serve.token_probs(x, float(u), min_p=min_p) for u in TEMPERATURES]
    sp.check()
    assert torch.isnan(got[:t]).all()
    want = torch.zeros((t, v), device="cuda")
    want[:, v - 1] = 1.0
    assert torch.equal(got[t:], want)
    for p in one:
        assert torch.isnan(p[:t]).all() and torch.equal(p[t:], want)


@pytest.mark.gpu
@pytest.mark.parametrize("v", [9, 40000])
def test_nothing_is_drawn_where_nothing_is_open(v):
    """A greedy request whose mask leaves nothing: no draft is kept, no token comes behind, and it is recorded."""
    from paper_2405_03594_gb300 import serve, sp

    def i32(*a):
        return torch.tensor(a, dtype=torch.int32, device="cuda")

    x = torch.full((3, v), -torch.inf, device="cuda")
    x[2, 4] = 1.0
    p = serve.token_probs(x, 0.0)
    ids = torch.zeros(3, dtype=torch.int64, device="cuda")  # the draft is token 0
    a, r, n = serve.verify_drafts(p, ids, i32(0, 2, 3), i32(1, 0), torch.zeros(3, device="cuda"), torch.zeros(2, device="cuda"))
    with pytest.raises(sp.SpError, match="INVALID_ARG"):
        sp.check()
    assert [a.tolist(), r.tolist(), n.tolist()] == [[0, 0], [1, 0], [-1, 4]]
    sp.check()
