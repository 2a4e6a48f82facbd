"""The 4-bit stack (paper_2505_23219_amd/q4_step.py): its quantiser, and its steps against a plain
forward pass in 64 bits over the weights and the cache rows that the library holds.

Tolerances.  The stack rounds about eight vectors a layer to fp16 (norms, q/k/v, turned q, attention's
probabilities and result, SwiGLU), each with a relative error of at most 2^-11 an entry.  The entries of
the two-layer stacks' logits have a deviation of 0.02 sqrt(256) = 0.32; sixteen independent roundings with
an r.m.s. of 2^-11 / sqrt(3) each leave 0.32 * 4 * 2.8e-4 = 3.6e-4, and six deviations with a factor of two
for what a layer amplifies are 4.3e-3: 5e-3 is allowed.  A cache row is off by half a step of its group
where the same value is quantised, plus the same 5e-3 where the value itself is off."""
import numpy as np
import pytest
import torch

import q4_plain as P
from paper_2505_23219_amd import binding as B, q4_step, workloads as wl

TOL = 5e-3


@pytest.mark.parametrize("N,K,group", [(3, 256, 32), (16, 688, 128), (5, 70, 64), (1, 2, 32)])
def test_quantised_weights_are_within_half_a_step(N, K, group):
    w = torch.from_numpy(np.random.default_rng(N * K).normal(0, 0.02, (N, K)).astype(np.float16))
    w[0, :2] = 0
    codes, scale, zero = q4_step.quantise_weight(w, group)
    assert codes.dtype == torch.uint8 and codes.shape == (N, K // 2)
    assert scale.dtype == torch.float16 and scale.shape == zero.shape == (N, -(-K // group))
    back = P.unpack_weight(codes.numpy(), scale.numpy(), zero.numpy(), K, group)
    step = np.repeat(scale.numpy().astype(np.float64), group, 1)[:, :K]
    # the last code of a group can be up to 15 * 2^-11 of a step short: the fp16 scale may have been rounded down
    assert (np.abs(back - w.numpy().astype(np.float64)) <= 0.51 * step).all()
    assert (back[0, :2] == 0).all()


def test_a_matrix_of_zeros_stays_one():
    codes, scale, zero = q4_step.quantise_weight(torch.zeros(4, 96), 64)
    assert (P.unpack_weight(codes.numpy(), scale.numpy(), zero.numpy(), 96, 64) == 0).all()


def _matrix(w, group):
    codes, scale, zero = q4_step.quantise_weight(w, group)
    return P.unpack_weight(codes.numpy(), scale.numpy(), zero.numpy(), w.shape[1], group)


def _norm(x, g, eps):
    return x / np.sqrt((x * x).mean(1, keepdims=True) + eps) * g.numpy().astype(np.float64)


def _forward(shape, nkv, group, layers, head, x, parent, kv_len, held_k, held_v):
    """Logits and per layer the new (keys, values) in 64 bits; attention reads the held rows."""
    M, d, rep = x.shape[0], shape.d, shape.nh // nkv
    pos, see = kv_len + P.depths(parent), P.sees_of_parent(parent)
    rows = []
    for i, w in enumerate(layers):
        qkv = _norm(x, w["g_attn"], shape.rms_eps) @ _matrix(q4_step.grouped_heads(w["Wqkv"], shape, nkv), group).T
        qkv = qkv.reshape(M, shape.nh + 2 * nkv, d)
        q = P.turn(qkv[:, :shape.nh], pos, shape.rope_base)
        rows.append((P.turn(qkv[:, shape.nh:shape.nh + nkv], pos, shape.rope_base), qkv[:, shape.nh + nkv:]))
        a, _ = P.attention(q, held_k[i], held_v[i], see, kv_len, d ** -0.5)
        x = x + a.reshape(M, -1) @ _matrix(w["Wo"], group).T
        gu = _norm(x, w["g_ffn"], shape.rms_eps) @ _matrix(w["Wgu"], group).T
        gate, up = gu[:, :shape.F], gu[:, shape.F:]
        x = x + (gate / (1 + np.exp(-gate)) * up) @ _matrix(w["Wdown"], group).T
    return _norm(x, head["g_final"], shape.rms_eps) @ _matrix(head["Wlm"], group).T, rows


@pytest.mark.gpu
@pytest.mark.parametrize("nkv,group,M", [(4, 128, 1), (2, 64, 9), (1, 32, 24), (4, 128, 70)])
def test_steps_with_commits_between(nkv, group, M):
    shape = wl.with_layers(wl.TINY, 2)
    layers = [wl.layer_weights(shape, 5, i) for i in range(2)]
    head = wl.head_weights(shape, 5)
    stack = q4_step.Q4Stack(shape, nkv, layers, head, 160, group)
    table = wl.embedding_table(shape, 5)
    parent = wl.tree_random(M, 5, M)
    tree = torch.from_numpy(parent).cuda()
    tokens = torch.from_numpy(wl.draft_tokens(M, shape.V, M)).cuda()
    kv_len = 0
    for step in range(3):
        logits = stack.step(B.ghd_embed(table.cuda(), tokens), tree, kv_len)
        held_k, held_v = (t.cpu().numpy() for t in B.ghd_kv_read_q4(stack.cache, 0, kv_len + M))
        want, rows = _forward(shape, nkv, group, layers, head, table[tokens.cpu().long()].numpy().astype(np.float64),
                              parent, kv_len, held_k, held_v)
        for i in range(2):
            for got, exact in ((held_k[i, kv_len:], rows[i][0]), (held_v[i, kv_len:], rows[i][1])):
                g = exact.reshape(M, -1, 32)
                half = np.repeat((g.max(-1) - g.min(-1)) / 30, 32, -1).reshape(exact.shape)
                assert (np.abs(got - exact) <= half + TOL).all(), (step, i)
        assert np.abs(logits.cpu().numpy() - want).max() <= TOL, step
        # the path to the deepest node is accepted, whatever the logits say
        depth = P.depths(parent)
        path, node = [], int(depth.argmax())
        while node >= 0:
            path.insert(0, node)
            node = int(parent[node])
        res = torch.tensor([len(path), 1] + path + [0] * (M - len(path)), dtype=torch.int32, device="cuda")
        stack.commit(res, M, kv_len)
        after = [t.cpu().numpy() for t in B.ghd_kv_read_q4(stack.cache, 0, kv_len + len(path))]
        for got, before in zip(after, (held_k, held_v)):
            assert np.array_equal(got[:, :kv_len], before[:, :kv_len])
            assert np.array_equal(got[:, kv_len:], before[:, [kv_len + n for n in path]])
        kv_len += len(path)
        tokens = tokens.roll(1)


@pytest.mark.gpu
def test_decoding_with_trees_takes_fewer_steps(capsys, monkeypatch):
    monkeypatch.setattr("sys.argv", ["q4_step", "--tokens", "24", "--kv-heads", "2", "--group", "64"])
    q4_step.main()
    one, trees = capsys.readouterr().out.strip().splitlines()
    assert "24 tokens in 24 steps" in one
    assert int(trees.split(" in ")[1].split()[0]) < 24
