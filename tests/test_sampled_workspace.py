"""The workspace of sampled acceptance without draft probabilities: what it takes, and nothing behind it."""
import pytest
import torch

import test_sparse_arguments as A
from paper_2505_23219_amd import binding as B


def test_a_call_without_draft_probabilities_takes_a_small_one():
    for M, V in ((1, 1), (8, 1000), (64, 32000), (128, 131072), (128, 262144)):
        small, whole = B.ghd_accept_sampled_undrawn_workspace_bytes(M, V), B.ghd_accept_sampled_workspace_bytes(M, V)
        assert 0 < small <= 400_000 and whole >= small + 8 * M * V
        assert A._accept(M=M, V=V, ws_bytes=small - 1) == A.WORKSPACE
        assert A._accept(M=M, V=V, ws=A.FAR[5] + 8, ws_bytes=small) == A.ALIGN            # (it is not the size that is refused)
        assert A._accept(M=M, V=V, ws=A.FAR[5] + 8, ws_bytes=small, q=A.FAR[14], rows=M) == A.WORKSPACE
        assert A._accept(M=M, V=V, ws=A.FAR[5] + 8, ws_bytes=whole, q=A.FAR[14], rows=M) == A.ALIGN
    for V in (1, 4096, 4097, 262144):
        sizes = [B.ghd_accept_sampled_undrawn_workspace_bytes(M, V) for M in range(1, 129)]
        assert sizes == sorted(sizes)
    for M, V in ((0, 10), (129, 10), (1, 0), (1, 262145)):
        assert B.ghd_accept_sampled_undrawn_workspace_bytes(M, V) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("M,V", [(1, 5), (9, 1001), (64, 32000), (128, 4097), (3, 262144)])
def test_nothing_behind_it_is_written(M, V):
    import test_gpu_sampled as S
    need = B.ghd_accept_sampled_undrawn_workspace_bytes(M, V)
    room = torch.full((need + 4096,), 255, dtype=torch.uint8, device="cuda")
    for seed in range(3):
        S._check(S._case(M, V, "random" if seed else "star", "none", seed), ws=room[2048:2048 + need])
        S._check(S._case(M, V, "chain", "none", seed))
    assert (room[:2048] == 255).all() and (room[2048 + need:] == 255).all()


@pytest.mark.gpu
def test_it_is_refused_where_drafts_have_probabilities():
    import test_gpu_sampled as S
    case = S._case(9, 1001, "random", "rows", 1)
    with pytest.raises(B.GhdError):
        S._gpu(case, ws=B.workspace(B.ghd_accept_sampled_undrawn_workspace_bytes(9, 1001)))
