"""Sizes of the routed contractions past 32 bits, on a machine without a GPU: the
index arithmetic of their kernels is compiled for the host and checked there, and
calls that no launch holds are refused before any HIP call (the addresses are
never read)."""
import os
import shutil
import subprocess

import pytest

from paper_2105_13480_amd import cnn

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
F32, BF16, OBF16 = cnn.CNN_F32, cnn.CNN_BF16, cnn.CNN_BF16_OBF16
OVERFLOW = -4
P = [i << 58 for i in range(1, 12)]  # addresses far from each other


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not installed")
def test_threads_past_31_bits(tmp_path):
    exe = str(tmp_path / "check")
    res = subprocess.run([HIPCC, "-O2", "-std=c++17", "-x", "hip", "--offload-arch=gfx950",
                          "-I", os.path.join(ROOT, "paper_2105_13480_amd", "csrc"),
                          os.path.join(ROOT, "tests", "routed_host", "check_unit_of_thread.cpp"), "-o", exe],
                         capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-4000:]
    run = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert run.returncode == 0 and "bad 0" in run.stdout, run.stdout + run.stderr


def test_adapted_rows_past_a_launch():
    """Few rows of so many features that the last launch would have 2^32 threads."""
    for Nt, Nk in ((352, 48806447), (17, 1011000000), (64, 1 << 28)):
        assert Nt * ((Nk + 3) // 4) >= 1 << 32
        assert cnn.lib().cnn_adapt_fwd(*P[:7], Nt, 8, Nk, 2, 4, BF16, P[8], 1 << 57, None) == OVERFLOW, (Nt, Nk)


def test_products_of_sizes_that_wrap():
    """Ker of 2^64 elements and more, which modulo 2^64 are none or few, and as many
    tiles: refused, also where Ker is NULL as only an empty tensor may be."""
    L = cnn.lib()
    for Ng, Nk, Nc in ((64, 1 << 29, 1 << 29), (256, 1 << 29, 1 << 27), (65535, (1 << 30) - 1, (1 << 30) - 1),
                       (32768, (1 << 30) - 1, (1 << 30) - 1)):
        for ker in (P[1], None):
            assert L.cnn_group_fwd(P[0], ker, P[2], P[3], P[4], 8, 16, Ng, Nc, Nk, BF16, None) == OVERFLOW
            assert L.cnn_group_bwd_in(P[0], ker, P[2], P[3], 16, Ng, Nc, Nk, BF16, None) == OVERFLOW
            assert L.cnn_group_bwd_ker(P[0], P[1], ker, P[3], P[4], 8, 16, Ng, Nc, Nk, BF16, None) == OVERFLOW


def test_more_threads_than_a_launch_holds():
    """2^32 threads: CNN_E_OVERFLOW, not an error of the launch.  The sizes fit the
    GPU's memory, or each of them its limit."""
    L, m = cnn.lib(), (1 << 30) - 1
    assert L.cnn_combine(*P[:4], 1 << 23, 1, 1 << 23, 4096, OBF16, None) == OVERFLOW
    assert L.cnn_combine(*P[:4], 1 << 24, 1, 1 << 23, 1024, F32, None) == OVERFLOW
    assert L.cnn_combine_bwd(*P[:7], 1 << 24, 1, 1 << 24, 2048, OBF16, None) == OVERFLOW
    assert L.cnn_combine_bwd(*P[:7], m, 4, 8, 2048, OBF16, None) == OVERFLOW  # weights' gradients alone
    assert L.cnn_route_bwd(*P[:5], 1 << 28, 8, 2, F32, 0, None) == OVERFLOW
    assert L.cnn_route_bwd(*P[:5], 1 << 26, 300, 2, F32, 0, None) == OVERFLOW
    for dtype in (F32, BF16, OBF16):
        for Nc in (8, 7):
            assert L.cnn_group_fwd(*P[:5], m, m, 1, Nc, 16, dtype, None) == OVERFLOW
            assert L.cnn_group_bwd_in(*P[:4], m, 1, 16, Nc, dtype, None) == OVERFLOW
            assert L.cnn_adapt_fwd(*P[:7], m, Nc, 16, 2, 4, dtype, P[8], 1 << 57, None) == OVERFLOW
        assert L.cnn_group_fwd(*P[:5], 65535, 65535, 65535, 1024, 8192, dtype, None) == OVERFLOW
        assert L.cnn_group_bwd_ker(*P[:5], 65535, 65535, 65535, 5000, 5000, dtype, None) == OVERFLOW
