"""What the 4-bit linear layer reads of x: nothing behind its last number.  Shown without a GPU: from the
arithmetic of the requests' offsets, and from the kernels' assembly, which has to leave that offset to the
hardware's check."""
import ctypes as C
import os
import re
import subprocess

import pytest

from paper_2505_23219_amd import binding as B, build


@pytest.mark.parametrize("M", [1, 2, 7, 8, 9, 16, 17, 31, 32, 33, 48, 63, 64, 65, 80, 96, 113, 128])
def test_requests_end_with_x_and_bring_all_of_it(M):
    out = (C.c_int64 * 2)()
    for N in (1, 1003, 22016):
        for K in (8, 64, 72, 128, 136, 1288, 4096):
            for ldx in (K, K + 8, K + 120, 4 * K + 1000, 1 << 16):
                B.lib().ghd_debug_q4_x(M, N, K, ldx, out)
                assert out[0] <= ((M - 1) * ldx + K) * 2, (N, K, ldx)
                assert out[1] == M * K, (N, K, ldx)
    K = 65536
    B.lib().ghd_debug_q4_x(M, 64, K, 1 << 23, out)
    assert out[0] <= ((M - 1) * (1 << 23) + K) * 2 and out[1] == M * K


def test_the_whole_offset_is_the_lanes(tmp_path):
    """The hardware checks the offset in a lane's register against the size of x; one in a scalar register may be left
    out of the check, so the loads of x must have none."""
    out = str(tmp_path / "q4_linear.s")
    flags = [f for f in build.FLAGS if not f.startswith("-Rpass") and f != "-fPIC"]
    subprocess.run([build._hipcc()] + flags + ["--cuda-device-only", "-S", os.path.join(build.CSRC, "q4_linear.hip"), "-o", out], check=True,
                   capture_output=True)
    loads = re.findall(r"^\s*buffer_load_\w+ (.*)$", open(out).read(), re.M)
    assert len(loads) > 100
    for load in loads:
        assert re.fullmatch(r"v\d+, s\[\d+:\d+\], 0 offen( offset:\d+)? lds", load), load
