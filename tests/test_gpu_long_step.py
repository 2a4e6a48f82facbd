"""A decoding loop over a long cache: bounds of blocks that become whole, selection, sparse attention of a drafted tree, logits, sampled
acceptance, commit - every step against the plain 64-bit forms."""
from types import SimpleNamespace

import pytest
import torch

import sparse_plain as P
import test_gpu_sparse as T
from paper_2505_23219_amd import binding as B, workloads as wl

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,nh,tree,drafts,T_", [(64, 4, "chain", False, 0.9), (128, 2, "random", False, 0.9), (64, 8, "star", True, 0.9),
                                                (128, 4, "random", True, 0.9), (64, 4, "chain", False, 0.05), (128, 2, "random", False, 0.1)])
def test_steps(d, nh, tree, drafts, T_):
    V, M, capacity, kv_len, count = 500, 12, 1024, 600, 4
    g = T._gen(d + nh)
    k, v, kd, vd = T._cache(nh, capacity, d, 7)
    parent = {"chain": wl.tree_chain(M), "star": wl.tree_star(M)}.get(tree, wl.tree_random(M, 4, 3)).tolist()
    pd, see = torch.tensor(parent, dtype=torch.int32, device="cuda"), P.ancestors(parent)
    W = (torch.randn(V, nh * d, generator=g) * 0.3).half()
    Wp = B.ghd_pack_weight(W.cuda())
    shape = wl.ModelShape("loop", nh * d, nh, d, 256, V, 1)
    stack = SimpleNamespace(cfg=B.make_cfg(shape, capacity), kv=(B.KV * 1)(B.KV(kd.data_ptr(), vd.data_ptr())))
    bounds, whole = B.BlockBounds(nh, d, capacity), 0
    ws = B.workspace(max(B.ghd_block_select_workspace_bytes(M, capacity, nh), B.ghd_sparse_attention_workspace_bytes(M, capacity - M, nh, nh, d),
                         B.ghd_accept_sampled_workspace_bytes(M, V)))
    committed = 0
    for step in range(14):
        rows = torch.randn(2, nh, M, d, generator=g).half()
        q, u = torch.randn(M, nh, d, generator=g).half(), torch.rand(M, generator=g)
        kd[:, kv_len:kv_len + M], vd[:, :, kv_len:kv_len + M] = rows[0].cuda(), rows[1].transpose(1, 2).cuda()
        if kv_len // 64 > whole:
            B.ghd_block_bounds(bounds, kd, whole, kv_len // 64 - whole)
            whole = kv_len // 64
        assert whole == kv_len // 64
        sel = B.ghd_block_select(q.cuda(), bounds, kv_len, count, ws=ws)
        out = B.ghd_sparse_attention(q.cuda(), kd, vd, sel, kv_len, parent=pd, ws=ws)
        logits = B.ghd_linear_skinny(out.view(M, nh * d), Wp, V)
        draft = logits + torch.randn(M, V, generator=g).cuda() if drafts else None
        tokens = torch.zeros(M, dtype=torch.int32)
        best = torch.sort((logits if draft is None else draft).cpu(), dim=1, descending=True, stable=True).indices
        for i in range(1, M):
            tokens[i] = best[parent[i], sum(parent[j] == parent[i] for j in range(i))]
        res = B.ghd_accept_sampled(logits, tokens.cuda(), pd, u.cuda(), T_, q_logits=draft, ws=ws)

        kc, vc = kd.cpu(), vd.cpu()
        chosen = P.select(P.scores(q, P.bounds(kc, whole)), count, 1, 1)
        assert torch.equal(sel.cpu(), P.words(chosen))
        want, size = P.attend(q, kc, vc, chosen, see, kv_len, d ** -0.5)
        off = (out.cpu().double() - want).abs()
        assert (off <= T._tolerance(size, want, q, kc[:, :kv_len + M], vc[:, :, :kv_len + M], d ** -0.5, kv_len + M)).all()
        path = P.accept(logits.cpu(), tokens, parent, u, T_, None if draft is None else draft.cpu())
        assert res.tolist()[:len(path)] == path

        B.ghd_commit_path(stack, res, M, kv_len)
        nodes = [kv_len + i for i in path[2:]]
        assert torch.equal(kd[:, kv_len:kv_len + path[0]].cpu(), kc[:, nodes]) and torch.equal(vd[:, :, kv_len:kv_len + path[0]].cpu(), vc[:, :, nodes])
        kv_len += path[0]
        committed += path[0]
    assert committed >= 14
    if T_ < 0.9:                                 # drafts were accepted
        assert committed > 28
    if tree == "chain" and T_ < 0.9:             # and a block became whole on the way
        assert kv_len // 64 > 600 // 64
