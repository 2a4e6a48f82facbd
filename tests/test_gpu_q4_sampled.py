"""Decoding with a 4-bit stack and sampled acceptance."""
import pytest
import torch

from paper_2505_23219_amd import binding as B, q4_step, workloads as wl

pytestmark = pytest.mark.gpu


def _stack(capacity=96):
    shape = wl.with_layers(wl.TINY, 2)
    layers = [wl.layer_weights(shape, 5, i) for i in range(2)]
    return q4_step.Q4Stack(shape, 2, layers, wl.head_weights(shape, 5), capacity, 64), wl.embedding_table(shape, 5, "cuda")


def _numbers(seed):
    return torch.Generator("cuda").manual_seed(seed)


def test_next_to_no_temperature_is_greedy():
    stack, table = _stack()
    greedy, _, _ = q4_step.decode(stack, table, 1, 20, [-1])
    sampled, _, _ = q4_step.decode(stack, table, 1, 20, [-1], temperature=1e-7, generator=_numbers(3))
    assert sampled == greedy


def test_a_seed_gives_its_tokens_and_drafts_are_taken():
    stack, table = _stack()
    parent = wl.tree_medusa(16, (4, 2, 1, 1), 1).tolist()

    def run(seed, T, draft=None):
        return q4_step.decode(stack, table, 1, 24, [-1] if draft is None else parent, draft, T, _numbers(seed))[:2]
    plain, steps = run(1, 0.8)
    assert (plain, steps) == run(1, 0.8) and plain != run(2, 0.8)[0] and steps == 24 and all(0 <= t < stack.shape.V for t in plain)
    # the likeliest tokens as drafts, at a temperature at which they mostly are what is sampled
    greedy = q4_step.decode(stack, table, 1, 40, [-1])[0]
    depth = [0] * len(parent)
    for i in range(1, len(parent)):
        depth[i] = depth[parent[i]] + 1
    tokens, steps = run(1, 1e-4, lambda written: [greedy[min(len(written) + depth[i] - 1, 39)] for i in range(1, len(parent))])
    assert steps < 24 and tokens[:16] == greedy[:16]


def test_the_command(capsys, monkeypatch):
    monkeypatch.setattr("sys.argv", ["q4_step", "--tokens", "16", "--kv-heads", "2", "--group", "64", "--temperature", "0.7", "--seed", "4"])
    q4_step.main()
    one, trees = capsys.readouterr().out.strip().splitlines()
    assert "16 tokens in 16 steps" in one and "trees of 16 nodes" in trees and "same" not in trees
