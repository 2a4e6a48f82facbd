"""What the Python calls of the 4-bit operators take and refuse."""
import os
import subprocess
import sys
from types import SimpleNamespace

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


def _cache(**kw):
    return SimpleNamespace(**{**dict(L=1, nkv=2, d=64, capacity=64, device=torch.device("cpu"), layers=[None], kv=None), **kw})


def _host_calls():
    """Calls with tensors in host memory, of wrong types or shapes."""
    half, byte, i32 = (lambda *n: torch.zeros(n, dtype=torch.float16)), (lambda *n: torch.zeros(n, dtype=torch.uint8)), (
        lambda *n: torch.zeros(n, dtype=torch.int32))
    Wq = byte(B.lib().ghd_weight_q4_bytes(16, 64, 32))
    ws = byte(1 << 16)
    cache, q, mask = _cache(), half(3, 4, 64), torch.zeros(3, 2, dtype=torch.int64)
    yield lambda: B.ghd_pack_weight_q4(byte(16, 32), half(16, 2), None, 32)
    yield lambda: B.ghd_linear_q4(half(2, 64), Wq, 16, 32, ws=ws)
    yield lambda: B.ghd_linear_q4(half(2, 64), Wq, 16, 32, ws=ws, y=torch.zeros(2, 17))
    yield lambda: B.ghd_kv_append_q4(cache, 0, half(3, 2, 64), half(3, 2, 64), 0)
    yield lambda: B.ghd_tree_attention_q4(q, cache, 0, i32(3), 0, ws=ws)
    yield lambda: B.ghd_tree_attention_q4(q, cache, 0, i32(4), 0, ws=ws)
    yield lambda: B.ghd_tree_attention_q4(q, _cache(d=128), 0, i32(3), 0, ws=ws)
    yield lambda: B.ghd_masked_attention_q4(q, cache, 0, mask, 0, ws=ws)
    yield lambda: B.ghd_masked_attention_q4(q, cache, 0, mask[:2], 0, ws=ws)
    yield lambda: B.ghd_commit_path_q4(cache, i32(5), 3, 0)
    yield lambda: B.ghd_kv_read_q4(cache, 0, 3)
    yield lambda: B.KvQ4(1, 2, 64, 64, "cpu")


def _refused():
    for i, call in enumerate(_host_calls()):
        try:
            call()
        except ValueError:
            continue
        raise SystemExit("call %d was not refused" % i)
    print("refused", i + 1)


def test_host_tensors_are_refused():
    _refused()


def test_they_are_refused_without_assertions_too():
    here = os.path.dirname(os.path.abspath(__file__))
    r = subprocess.run([sys.executable, "-O", "-c", "import test_q4_arguments as t; t._refused()"], capture_output=True, text=True,
                       env={**os.environ, "PYTHONPATH": os.pathsep.join([here, os.path.dirname(here)])})
    assert r.returncode == 0 and "refused 12" in r.stdout, r.stdout + r.stderr


@pytest.mark.gpu
def test_workspaces():
    """Any type, by its bytes; on the GPU and in one piece."""
    Wq, x = _matrix(4096, 4096), torch.randn(32, 4096, device="cuda").half()
    n = B.ghd_linear_q4_workspace_bytes(32, 4096, 4096)
    want = B.ghd_linear_q4(x, Wq, 4096, 32)
    assert torch.equal(B.ghd_linear_q4(x, Wq, 4096, 32, ws=torch.empty(-(-n // 4), device="cuda")), want)
    room = torch.empty((2, n), dtype=torch.uint8, device="cuda")
    for ws in (room[0].cpu(), room.t()):
        with pytest.raises(ValueError):
            B.ghd_linear_q4(x, Wq, 4096, 32, ws=ws)
    cache = B.KvQ4(1, 2, 64, 64)
    q, parent = torch.randn(3, 4, 64, device="cuda").half(), torch.tensor([-1, 0, 1], dtype=torch.int32, device="cuda")
    for ws in (room[0].cpu(), room.t()):
        with pytest.raises(ValueError):
            B.ghd_tree_attention_q4(q, cache, 0, parent, 5, ws=ws)
    for bad in (q.float(), q.transpose(0, 1)):
        with pytest.raises(ValueError):
            B.ghd_tree_attention_q4(bad, cache, 0, parent, 5)
    for bad in (q[:, :1], q[:, ::2].float(), q[:, ::2], q[:, :2].transpose(1, 2)):
        with pytest.raises(ValueError):
            B.ghd_kv_append_q4(cache, 0, bad, q[:, :2], 5)
