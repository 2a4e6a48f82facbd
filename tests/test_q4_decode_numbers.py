"""What the 4-bit decoding loop refuses, and that it ends where no token can be sampled (the library's calls replaced by plain ones)."""
import math
from types import SimpleNamespace

import pytest
import torch

from paper_2505_23219_amd import q4_step


class _Stack:
    """Logits of ten tokens; from step `bad` on none is a number."""

    def __init__(self, bad):
        self.shape, self.bad, self.at, self.committed = SimpleNamespace(V=10), bad, 0, 0

    def step(self, x, tree, kv_len):
        self.at += 1
        return torch.full((1, 10), math.nan) if self.at > self.bad else torch.arange(10.0)[None]

    def commit(self, res, M, kv_len):
        self.committed += 1


def _accept_sampled(logits, tokens, parent, u, temperature, res, ws):
    res.copy_(torch.tensor([1, -1 if torch.isnan(logits).all() else int(logits[0].argmax()), 0]))


def _accept_greedy(logits, tokens, parent, res, amax):
    res.copy_(torch.tensor([1, int(logits[0].argmax()), 0]))


@pytest.fixture
def plain(monkeypatch):
    monkeypatch.setattr(q4_step, "B", SimpleNamespace(
        ghd_embed=lambda table, nodes: table[nodes.long()], ghd_accept_greedy_static=_accept_greedy, ghd_accept_sampled=_accept_sampled,
        ghd_accept_sampled_undrawn_workspace_bytes=lambda M, V: 256, workspace=lambda n, device: torch.zeros(n)))
    monkeypatch.setattr(torch.cuda, "synchronize", lambda: None)


def test_a_token_that_cannot_be_drawn_ends_it(plain):
    table = torch.zeros(10, 4)
    assert q4_step.decode(_Stack(99), table, 1, 5, [-1], temperature=0.5)[:2] == ([9] * 5, 5)
    with pytest.raises(FloatingPointError, match="behind the 3"):
        q4_step.decode(_Stack(3), table, 1, 5, [-1], temperature=0.5)
    with pytest.raises(FloatingPointError, match="behind the 0"):
        q4_step.decode(_Stack(0), table, 1, 5, [-1], temperature=2.0)


@pytest.mark.parametrize("temperature", [-1.0, -1e-30, math.nan, math.inf, -math.inf])
def test_temperatures_that_are_none(plain, temperature):
    with pytest.raises(ValueError, match="temperature"):
        q4_step.decode(_Stack(99), torch.zeros(10, 4), 1, 5, [-1], temperature=temperature)


def test_greedy_as_before(plain):
    assert q4_step.decode(_Stack(99), torch.zeros(10, 4), 1, 4, [-1])[:2] == ([9] * 4, 4)
    assert q4_step.decode(_Stack(99), torch.zeros(10, 4), 1, 4, [-1], temperature=-0.0)[:2] == ([9] * 4, 4)
