"""Temperatures go to rows, one each: a vector of any other length is refused, not read from its beginning (CPU: tensors that
say they are on a GPU stand in for those that are)."""
import pytest
import torch

from paper_2405_03594_gb300 import serve
from tests.test_serve_devices import Stream, gpu


@pytest.fixture(autouse=True)
def _current(monkeypatch):
    monkeypatch.setattr(serve, "_current_device", lambda: 0)


@pytest.mark.parametrize("n", [0, 1, 2, 4, 64])
def test_as_many_temperatures_as_rows(n):
    """Of a step with three rows, one per request where four have a place: a vector of four is the requests', not the rows'."""
    out = gpu(torch.zeros((3, 10)))
    with pytest.raises(ValueError, match="temperature"):
        serve.token_probs(gpu(torch.zeros((3, 10))), gpu(torch.ones(n)), out=out, stream=Stream)


def test_a_temperature_of_one_row_is_no_number():
    for bad in (torch.ones(()), torch.ones((3, 1)), torch.ones(3).double(), torch.ones(6)[::2]):
        with pytest.raises(ValueError, match="temperature"):
            serve.token_probs(gpu(torch.zeros((3, 10))), gpu(bad), out=gpu(torch.zeros((3, 10))), stream=Stream)
