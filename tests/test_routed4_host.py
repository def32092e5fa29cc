"""Index arithmetic of the products with a Ker in 4 bits, compiled for the host and
checked there."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"

pytestmark = pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not installed")


def _run(tmp_path, name, lines=()):
    exe = str(tmp_path / "check")
    res = subprocess.run([HIPCC, "-O2", "-std=c++17", "-x", "hip", "--offload-arch=gfx950", "--cuda-host-only",
                          "-I", os.path.join(ROOT, "paper_2105_13480_amd", "csrc"), "-I", os.path.join(ROOT, "include"),
                          os.path.join(ROOT, "tests", "routed_host", name + ".cpp"), "-o", exe],
                         capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-4000:]
    return subprocess.run([exe], input="".join(" ".join(map(str, l)) + "\n" for l in lines), capture_output=True,
                          text=True, timeout=120)


def test_half_blocks_lie_within_their_row(tmp_path):
    """No byte of codes or scales past a row's end is read: rows of one block, where a
    stage has four half blocks and the row two, among them."""
    run = _run(tmp_path, "check_half_blocks")
    assert run.returncode == 0 and "bad 0" in run.stdout, run.stdout + run.stderr


def test_every_kernel_has_exact_cases(tmp_path):
    """The calls of the GPU tests reach every kernel that the choice has, by the choice
    itself: the forward products' tests, the small and long ones with tensors at whole
    units and at odd elements, and those of each kernel."""
    import test_gpu_group4 as listed
    import test_gpu_group4_reach as reach

    def calls(cases, starts):
        for case in cases:
            Nt, Ng, active, Kt, _, Nc, Nk = case
            for element, byte in starts(Nt):
                for gathered in (1, 0):
                    Np = Nt * min(Kt, active)
                    yield (Nt if gathered else Np, Np, Ng, Nc, Nk, gathered, 2 * element, byte, byte)

    odd = lambda Nt: [(Nt % 2, int(Nt % 4 > 0))]  # noqa: E731
    both = lambda Nt: [(i, i) for i in reach.START]  # noqa: E731
    none = lambda Nt: [(0, 0)]  # noqa: E731

    def picks(lines):
        run = _run(tmp_path, "pick_group4", lines)
        assert run.returncode == 0, run.stderr
        return [tuple(map(int, line.split())) for line in run.stdout.splitlines()]

    whole = [list(range(-1, 8)), list(range(-1, 6)), list(range(-1, 4)), [0, 2, 4]]
    exact = picks([*calls(listed.CASES, odd), *calls(reach.SMALL + reach.FEW, both)])
    assert [sorted(set(p)) for p in zip(*exact)] == whole
    kinds = picks(calls(reach.KINDS, none))
    assert [sorted(set(p)) for p in zip(*kinds)] == whole
