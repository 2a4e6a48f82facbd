"""A result of the 4-bit linear layer that meets its input or its weights is refused, one that lies between the input's
rows is not."""
import ctypes as C

import pytest
import torch

from paper_2505_23219_amd import binding as B

AT = 1 << 20


def _meets(y, x, W=1 << 40, M=16, N=64, K=128, ldx=None, ldy=None, out16=True):
    fn = B.lib().ghd_debug_q4_linear_meets
    fn.argtypes = [C.c_void_p] * 3 + [C.c_int] * 4 + [C.c_int64] * 2 + [C.c_uint32]
    return fn(y, x, W, M, N, K, 32, ldx or K, ldy or N, B.GHD_OUT_F16 if out16 else B.GHD_OUT_F32)


@pytest.mark.parametrize("out16", [True, False])
@pytest.mark.parametrize("M", [1, 2, 128])
def test_where_y_meets_x(M, out16):
    x, N, K = AT, 64, 128
    y_bytes, x_bytes = M * N * (2 if out16 else 4), M * K * 2
    for y, meets in [(x, 1), (x - y_bytes, 0), (x - y_bytes + 16, 1), (x + x_bytes, 0), (x + x_bytes - 16, 1), (x + x_bytes // 2, 1)]:
        assert _meets(y, x, M=M, out16=out16) == meets, y - x


def test_rows_between_rows():
    wide = 128 + 64                                                  # columns of one fp16 buffer: x, then y
    assert _meets(AT + 256, AT, ldx=wide, ldy=wide) == 0
    assert _meets(AT, AT + 128, ldx=wide, ldy=wide) == 0             # y first
    assert _meets(AT + 256 - 16, AT, ldx=wide, ldy=wide) == 1
    assert _meets(AT + 256, AT, ldx=wide, ldy=wide + 8) == 1         # rows of y creep into those of x
    assert _meets(AT + 256, AT, ldx=wide, ldy=wide // 2, out16=False) == 1
    # between the rows behind the first of few
    assert _meets(AT + 4096 - 128, AT, M=3, ldx=2048, ldy=2048) == 0


def test_where_y_meets_the_weights():
    n = B.lib().ghd_weight_q4_bytes(64, 128, 32)
    for y, meets in [(AT, 1), (AT + n - 16, 1), (AT + n, 0), (AT - 16 * 64 * 2, 0), (AT - 16 * 64 * 2 + 16, 1)]:
        assert _meets(y, 1 << 40, W=AT) == meets


def test_such_a_call_is_refused():
    assert B.lib().ghd_linear_q4(AT, AT, 1 << 40, 16, 64, 64, 32, 64, 64, B.GHD_OUT_F16, 1 << 41, 1 << 30, None) == B.GHD_ERR_SHAPE


@pytest.mark.gpu
def test_result_beside_its_input():
    torch.manual_seed(1)
    M, N, K, group = 33, 96, 256, 64
    codes = torch.randint(0, 256, (N, K // 2), dtype=torch.uint8, device="cuda")
    Wq = B.ghd_pack_weight_q4(codes, torch.rand(N, K // group, device="cuda").half(), None, group)
    wide = torch.randn(M, K + N, device="cuda").half()
    want = B.ghd_linear_q4(wide[:, :K].contiguous(), Wq, N, group, torch.float16)
    x = wide[:, :K].clone()
    assert torch.equal(B.ghd_linear_q4(wide[:, :K], Wq, N, group, y=wide[:, K:]), want)
    assert torch.equal(wide[:, :K], x) and torch.equal(wide[:, K:], want)
    with pytest.raises(B.GhdError):
        B.ghd_linear_q4(wide[:, :K], Wq, N, group, y=wide[:, K - 8:K - 8 + N])
    assert torch.equal(wide[:, :K], x)
