"""Probabilities of a row alone and among others: the kernel takes a row by one CTA or by several, as the number of rows goes, so
that the order of the sum differs; either is held to the bound of tests/test_gpu_drafts.py against 64 bits."""
import pytest
import torch

from tests.test_gpu_drafts import _check_probs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("v", [4096, 32000, 40001])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_a_row_alone_and_among_others(v, dtype):
    from paper_2405_03594_gb300 import serve, sp

    g = torch.Generator(device="cuda").manual_seed(v)
    x = (3 * torch.randn((320, v), generator=g, device="cuda")).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    t = (0.3 + torch.rand(320, generator=g, device="cuda"))
    among = serve.token_probs(x, t, min_p=0.001)
    assert torch.equal(serve.token_probs(x, t, min_p=0.001), among)
    for n in (1, 5, 40, 90, 160):
        for r in (0, 7, 160):
            some = serve.token_probs(x[r:r + n], t[r:r + n], min_p=0.001)
            assert torch.equal(serve.token_probs(x[r:r + n], t[r:r + n], min_p=0.001), some)
            rows = slice(r, r + min(n, 3))
            for p in (some[:min(n, 3)], among[rows]):
                _check_probs(p, x[rows].float().cpu().numpy(), t[rows].cpu().numpy(), 0.001)
            # (entries are left out by their own logit and the best one, which no order changes)
            assert torch.equal(some == 0, among[r:r + n] == 0)
    sp.check()


def test_temperatures_beside_the_results():
    """Right before the first entry and right behind the last one is no overlap."""
    from paper_2405_03594_gb300 import serve, sp

    x = torch.randn((3, 100), generator=torch.Generator(device="cuda").manual_seed(0), device="cuda")
    one = torch.full((3 + 300 + 3,), 0.5, device="cuda")
    want = serve.token_probs(x, 0.5)
    for t in (one[:3], one[303:]):
        assert torch.equal(serve.token_probs(x, t, out=one[3:303].view(3, 100)), want)
        assert (t == 0.5).all()
    with pytest.raises(sp.SpError, match="INVALID_ARG"):
        serve.token_probs(x, one[302:305], out=one[3:303].view(3, 100))
    sp.check()
