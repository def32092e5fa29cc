"""Index arithmetic of the products with a Ker in 4 bits, compiled for the host and
checked there."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"

pytestmark = pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not installed")


def _run(tmp_path, name):
    exe = str(tmp_path / "check")
    res = subprocess.run([HIPCC, "-O2", "-std=c++17", "-x", "hip", "--offload-arch=gfx950", "--cuda-host-only",
                          "-I", os.path.join(ROOT, "paper_2105_13480_amd", "csrc"), "-I", os.path.join(ROOT, "include"),
                          os.path.join(ROOT, "tests", "routed_host", name + ".cpp"), "-o", exe],
                         capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-4000:]
    return subprocess.run([exe], capture_output=True, text=True, timeout=120)


def test_half_blocks_lie_within_their_row(tmp_path):
    """No byte of codes or scales past a row's end is read: rows of one block, where a
    stage has four half blocks and the row two, among them."""
    run = _run(tmp_path, "check_half_blocks")
    assert run.returncode == 0 and "bad 0" in run.stdout, run.stdout + run.stderr
