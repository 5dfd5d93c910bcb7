"""Decoder.sample and Decoder.verify look at their arguments before the step changes the tables: a call that they refuse can be made
again (CPU: tensors that say they are on a GPU, and a step that only says that it was reached)."""
import math
import types

import pytest
import torch

from paper_2405_03594_gb300 import decoder, serve, sp
from tests.test_serve_devices import gpu

T, V, B = 5, 10, 2


class Reached(Exception):
    pass


class Ids(torch.Tensor):
    """Host ids; a Decoder compares where they are with where its rows are."""


@pytest.fixture
def dec(monkeypatch):
    monkeypatch.setattr(serve, "_current_device", lambda: 0)
    d = decoder.Decoder.__new__(decoder.Decoder)
    d.h = gpu(torch.zeros((8, 4), dtype=torch.bfloat16))
    d.head = types.SimpleNamespace(n=V)
    c = serve.KvCache(4, 2, 64, 16, data=torch.zeros(4 * 2 * 16 * 72, dtype=torch.uint8))
    d.batch = serve.Batch(c, 4, B, 8, 1)
    d.batch.__dict__["_gpu"] = 0

    def step(*_):
        raise Reached

    d.step = step
    return d


def _common():
    return dict(ids=gpu(torch.zeros(T, dtype=torch.int64)), new=gpu(torch.tensor([3, 2], dtype=torch.int32)), max_new=3,
                sample=gpu(torch.zeros(B)), temperature=gpu(torch.ones(T)), min_p=0.1)


def _drafts():
    return dict(drafts=gpu(torch.ones(B, dtype=torch.int32)), accept=gpu(torch.zeros(T)), draft_probs=gpu(torch.zeros((T, V))))


BAD = [("temperature", gpu(torch.ones(T - 1))), ("temperature", gpu(torch.ones(T + 1))), ("temperature", torch.ones(T)), ("temperature", math.nan),
       ("temperature", gpu(torch.ones(T).double())), ("min_p", -0.1), ("min_p", 1.5), ("min_p", math.nan), ("sample", torch.zeros(B)),
       ("sample", gpu(torch.zeros(B - 1))), ("sample", gpu(torch.zeros(B).double())), ("sample", gpu(torch.zeros(2 * B))[::2])]
BAD_DRAFTS = [("drafts", gpu(torch.ones(B - 1, dtype=torch.int32))), ("drafts", gpu(torch.ones(B, dtype=torch.int64))),
              ("drafts", torch.ones(B, dtype=torch.int32)), ("accept", gpu(torch.zeros(T - 1))), ("accept", torch.zeros(T)),
              ("accept", gpu(torch.zeros(T).bfloat16())), ("draft_probs", gpu(torch.zeros((T, V - 1)))), ("draft_probs", gpu(torch.zeros((T + 1, V)))),
              ("draft_probs", torch.zeros((T, V))), ("draft_probs", gpu(torch.zeros((T, V)).half())),
              ("draft_probs", gpu(torch.zeros((V, T)).t())), ("draft_probs", gpu(torch.zeros((1, V)).expand(T, V)))]


def test_good_arguments_reach_the_step(dec):
    for temperature in (gpu(torch.ones(T)), 0.7, 0, math.inf):
        with pytest.raises(Reached):
            dec.sample(**{**_common(), "temperature": temperature})
        for draft_probs in (_drafts()["draft_probs"], None, gpu(torch.zeros((T, V + 3)).bfloat16())[:, :V]):
            with pytest.raises(Reached):
                dec.verify(**{**_common(), "temperature": temperature}, **{**_drafts(), "draft_probs": draft_probs})


@pytest.mark.parametrize("name,value", BAD)
def test_a_sample_is_refused_before_the_step(dec, name, value):
    with pytest.raises((ValueError, sp.SpError)):
        dec.sample(**{**_common(), name: value})


@pytest.mark.parametrize("name,value", BAD + BAD_DRAFTS)
def test_a_verification_is_refused_before_the_step(dec, name, value):
    with pytest.raises((ValueError, sp.SpError)):
        dec.verify(**{**_common(), **_drafts(), name: value})


def test_a_vocabulary_that_nothing_is_drawn_from_is_refused_before_the_step(dec):
    dec.head.n = (1 << 22) + 1
    for call in (lambda: dec.sample(**_common()), lambda: dec.verify(**_common(), **{**_drafts(), "draft_probs": None})):
        with pytest.raises(sp.SpError, match="UNSUPPORTED"):
            call()
