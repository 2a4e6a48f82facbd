"""What the Python calls of the 4-bit operators take and refuse."""
import pytest
import torch

from paper_2505_23219_amd import binding as B


def _matrix(N=40, K=64, group=32):
    torch.manual_seed(3)
    codes = torch.randint(0, 256, (N, K // 2), dtype=torch.uint8, device="cuda")
    return B.ghd_pack_weight_q4(codes, torch.rand(N, -(-K // group), device="cuda").half(), None, group)


@pytest.mark.gpu
@pytest.mark.parametrize("step", [67, 64, (1 << 23) + 8])
def test_the_stride_of_a_single_row_says_nothing(step):
    Wq = _matrix()
    x = torch.randn(1, 64, device="cuda").half()
    want = B.ghd_linear_q4(x, Wq, 40, 32)
    apart = x.clone().as_strided((1, 64), (step, 1))
    y = torch.zeros(1, 40, device="cuda").as_strided((1, 40), (step % 40, 1))
    assert torch.equal(B.ghd_linear_q4(apart, Wq, 40, 32, y=y), want) and torch.equal(y, want)
