"""A row's result of the 4-bit linear layer does not depend on what the rows beside it hold."""
import pytest
import torch

from paper_2505_23219_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N,K,group", [(4096, 11008, 64), (1003, 1288, 32), (22016, 4096, 128), (64, 136, 32)])
@pytest.mark.parametrize("M", [2, 16, 40, 64, 75, 128])
def test_rows_beside(M, N, K, group):
    """To the bit, with as many rows (their number decides how k is cut)."""
    print("q4 rows beside", M, N, K, group, flush=True)
    torch.manual_seed(M + N)
    codes = torch.randint(0, 256, (N, K // 2), dtype=torch.uint8, device="cuda")
    scales = (torch.rand(N, -(-K // group), device="cuda") * 0.01).half()
    Wq = B.ghd_pack_weight_q4(codes, scales, None, group)
    x = torch.randn(M, K, device="cuda").half()
    want = B.ghd_linear_q4(x, Wq, N, group)
    for kept in sorted({0, M // 2, M - 1}):
        other = torch.randn(M, K, device="cuda").half() * 100
        other[kept] = x[kept]
        assert torch.equal(B.ghd_linear_q4(other, Wq, N, group)[kept], want[kept])
        other[[i for i in range(M) if i != kept]] = float("nan")
        assert torch.equal(B.ghd_linear_q4(other, Wq, N, group)[kept], want[kept])
