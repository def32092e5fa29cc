"""Products with Ker (and rows) in 4 bits on every kernel that the choice has (which one
takes a call is asked on the host, tests/test_routed4_host.py): the smallest contractions,
few rows of long ones, scales at the ends of their range, rows that are not in In and
offsets that are no order.

All against the definition in 64 bits on the CPU.  Values are whole numbers times powers
of two, so that no sum leaves fp32 and results are exact."""
import math

import pytest
import torch

import four_bits
from gpu_helpers import say
from paper_2105_13480_amd import routed
from test_gpu_group4 import OUT, _at, _order, _out, _product, _whole

pytestmark = pytest.mark.gpu

# (Nt, Ng, active, Kt, drop, Nc, Nk): contractions shorter than a unit of 16 bytes, of a unit,
# and of one block, with several tiles, groups, rows without a group
SMALL = [(9, 3, 3, 2, 0.2, 7, 5), (33, 2, 2, 1, 0.0, 2, 70), (40, 3, 2, 1, 0.1, 8, 130), (70, 4, 3, 2, 0.0, 31, 33),
         (5, 2, 2, 1, 0.0, 32, 7), (3, 2, 2, 1, 0.0, 1, 3), (50, 3, 3, 1, 0.1, 5, 6), (20, 2, 2, 1, 0.0, 16, 2),
         (130, 3, 2, 2, 0.1, 33, 4), (300, 2, 2, 1, 0.1, 24, 1), (257, 1, 1, 1, 0.0, 6, 200), (1, 1, 1, 1, 0.0, 9, 8)]
# rows of 53 to 63 blocks, and of 64 and more, that end with a block and within one
FEW = [(1, 1, 1, 1, 0.0, 1792, 250), (3, 1, 1, 1, 0.3, 1800, 100), (5, 2, 2, 1, 0.2, 1720, 33), (17, 1, 1, 1, 0.0, 1960, 15),
       (40, 2, 2, 1, 0.1, 2008, 1001), (2, 1, 1, 1, 0.0, 2048, 40), (6, 3, 2, 1, 0.0, 2056, 18), (4, 1, 1, 2, 0.0, 4072, 16)]
# one of each kernel at least
KINDS = [(40, 3, 2, 1, 0.05, 64, 40), (20, 2, 2, 1, 0.1, 7, 5), (5, 2, 2, 1, 0.2, 1792, 33), (6, 3, 2, 1, 0.0, 2056, 18),
         (70, 70, 66, 1, 0.0, 520, 40), (4100, 1, 1, 1, 0.01, 520, 8), (4100, 3, 2, 1, 0.02, 512, 104),
         (3000, 2, 2, 1, 0.02, 64, 264), (400, 5, 4, 1, 0.1, 64, 3000), (4100, 1, 1, 1, 0.02, 512, 2056),
         (4100, 2, 2, 1, 0.02, 2056, 128), (3000, 3, 3, 1, 0.05, 1000, 8), (9, 2, 2, 1, 0.1, 2049, 48), (9, 2, 2, 1, 0.0, 20, 9),
         (1000, 1, 1, 1, 0.0, 64, 2056)]
START = (0, 1)  # In's and dOut's first element, and the first byte of the scales


@pytest.mark.parametrize("out", OUT)
@pytest.mark.parametrize("start", START)
@pytest.mark.parametrize("case", SMALL + FEW, ids=str)
def test_small_and_long(case, start, out):
    say(f"[reach4] {case} {start} {out}")
    Nt, Ng, active, Kt, drop, Nc, Nk = case
    gen = torch.Generator().manual_seed(7 * Nt + Nc)
    offsets, rows = _order(gen, Nt, Ng, active, Kt, drop)
    Np, at = rows.numel(), rows.long().clamp_min(0)
    codes, scales = four_bits.random(gen, Ng, Nk, Nc=Nc)
    xc, xs = four_bits.random(gen, Nt, Nc=Nc)
    x, d = _whole(gen, Nt, Nc), _whole(gen, Np, Nk)
    ker = four_bits.values(codes, scales, Nc)
    k, s, o, r = codes.cuda(), _at(scales, start), offsets.cuda(), rows.cuda()

    def run(f, n):
        got = _out(Np + 1, n, OUT[out])
        f(got[:Np])
        assert torch.isnan(got[Np]).all()
        return got[:Np].cpu()

    want = _product(x.double()[at], ker, offsets).to(OUT[out])
    assert torch.equal(run(lambda t: routed.group_fwd4(_at(x, start), k, s, t, o, r), Nk), want)
    assert torch.equal(run(lambda t: routed.group_fwd4(_at(x[at], start), k, s, t, o), Nk), want)
    want = _product(four_bits.values(xc, xs, Nc)[at], ker, offsets).to(OUT[out])
    assert torch.equal(run(lambda t: routed.group_fwd4(xc.cuda(), k, s, t, o, r, InScales=_at(xs, start)), Nk), want)
    assert torch.equal(run(lambda t: routed.group_fwd4(xc[at].cuda(), k, s, t, o, InScales=_at(xs[at], start)), Nk), want)
    want = _product(d.double(), ker.transpose(1, 2).contiguous(), offsets).to(OUT[out])
    assert torch.equal(run(lambda t: routed.group_bwd_in4(_at(d, start), k, s, t, o), Nc), want)


# Ker's lowest scale byte of three and the power of two that bf16 values beside it are times:
# Ker's values down to 2^-128, which is subnormal in bf16, and up to 6 2^125; bf16 values
# that are subnormal
BESIDE = [(0, 100), (250, -100), (250, -133)]
# Ker's and In's lowest scale bytes
BOTH = [(0, 200), (200, 0), (252, 20), (20, 252), (0, 252)]


@pytest.mark.parametrize("out", OUT)
@pytest.mark.parametrize("low,power", BESIDE)
@pytest.mark.parametrize("case", KINDS, ids=str)
def test_scales_beside_bf16(case, low, power, out):
    """Products of the exact values, also where an operand is subnormal in bf16."""
    say(f"[scales4] {case} {low} {power} {out}")
    Nt, Ng, active, Kt, drop, Nc, Nk = case
    gen = torch.Generator().manual_seed(Nt + Nk)
    offsets, rows = _order(gen, Nt, Ng, active, Kt, drop)
    Np, at = rows.numel(), rows.long().clamp_min(0)
    codes, scales = four_bits.random(gen, Ng, Nk, Nc=Nc, low=low, high=low + 3)
    ker = four_bits.values(codes, scales, Nc)
    x, d = (_whole(gen, *n).double() * 2.0 ** power for n in ((Nt, Nc), (Np, Nk)))
    assert torch.equal(x.bfloat16().double(), x)
    k, s, o, r = codes.cuda(), scales.cuda(), offsets.cuda(), rows.cuda()
    want = _product(x[at], ker, offsets).to(OUT[out])
    assert torch.equal(routed.group_fwd4(x.bfloat16().cuda(), k, s, _out(Np, Nk, OUT[out]), o, r).cpu(), want)
    want = _product(d, ker.transpose(1, 2).contiguous(), offsets).to(OUT[out])
    assert torch.equal(routed.group_bwd_in4(d.bfloat16().cuda(), k, s, _out(Np, Nc, OUT[out]), o).cpu(), want)


@pytest.mark.parametrize("out", OUT)
@pytest.mark.parametrize("low,beside", BOTH)
@pytest.mark.parametrize("case", KINDS, ids=str)
def test_scales_of_both(case, low, beside, out):
    """Each value by itself may be past bf16's and fp32's range."""
    say(f"[scales44] {case} {low} {beside} {out}")
    Nt, Ng, active, Kt, drop, Nc, Nk = case
    gen = torch.Generator().manual_seed(Nt + Nk)
    offsets, rows = _order(gen, Nt, Ng, active, Kt, drop)
    Np, at = rows.numel(), rows.long().clamp_min(0)
    codes, scales = four_bits.random(gen, Ng, Nk, Nc=Nc, low=low, high=low + 3)
    xc, xs = four_bits.random(gen, Nt, Nc=Nc, low=beside, high=beside + 3)
    want = _product(four_bits.values(xc, xs, Nc)[at], four_bits.values(codes, scales, Nc), offsets).to(OUT[out])
    got = routed.group_fwd4(xc.cuda(), codes.cuda(), scales.cuda(), _out(Np, Nk, OUT[out]), offsets.cuda(), rows.cuda(),
                            InScales=xs.cuda())
    assert torch.equal(got.cpu(), want)


@pytest.mark.parametrize("case", KINDS, ids=str)
def test_infinite_ker_beside_bf16(case):
    """Ker's values of 2^128 and more are infinite: with zeros of In NaN, else infinite or,
    of both signs, NaN.  In is so small that no finite product or sum is; these are within
    the bound of an fp32 sum."""
    say(f"[infinite4] {case}")
    Nt, Ng, active, Kt, drop, Nc, Nk = case
    gen = torch.Generator().manual_seed(Nt)
    offsets, rows = _order(gen, Nt, Ng, active, Kt, drop)
    Np, at = rows.numel(), rows.long().clamp_min(0)
    codes, scales = four_bits.random(gen, Ng, Nk, Nc=Nc, low=252, high=255)
    keep = torch.rand(scales.shape, generator=gen) < 0.9
    scales[keep] = 200
    ker = four_bits.values(codes, scales, Nc).bfloat16().double()
    x, d = (_whole(gen, *n).double() * 2.0 ** -100 for n in ((Nt, Nc), (Np, Nk)))
    k, s, o, r = codes.cuda(), scales.cuda(), offsets.cuda(), rows.cuda()
    for got, v, w in ((routed.group_fwd4(x.bfloat16().cuda(), k, s, _out(Np, Nk, torch.float32), o, r), x[at], ker),
                      (routed.group_bwd_in4(d.bfloat16().cuda(), k, s, _out(Np, Nc, torch.float32), o), d, ker.transpose(1, 2).contiguous())):
        got, want = got.cpu().double(), _product(v, w, offsets)
        odd = ~torch.isfinite(want)
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        assert torch.equal(got[odd & ~torch.isnan(want)], want[odd & ~torch.isnan(want)])
        tol = (v.shape[1] + 8) * 2.0 ** -24 * _product(v.abs(), w.abs(), offsets)
        assert ((got - want).abs() <= tol)[~odd].all()


@pytest.mark.parametrize("case", KINDS, ids=str)
def test_rows_not_there_and_no_order(case):
    """Rows outside In read as zeros; of offsets that are no order no tile is run, so that
    results stay as they were."""
    say(f"[outside4] {case}")
    Nt, Ng, active, Kt, drop, Nc, Nk = case
    gen = torch.Generator().manual_seed(Nt + 1)
    offsets, rows = _order(gen, Nt, Ng, active, Kt, drop)
    Np = rows.numel()
    strange = torch.tensor([Nt, -1, Nt + 1, 1 << 30, -(1 << 31), (1 << 31) - 1], dtype=torch.int32)
    away = torch.rand(Np, generator=gen) < 0.2
    away[0] = away[Np // 2] = True
    rows[away] = strange[torch.randint(0, 6, (int(away.sum()),), generator=gen)]
    there = ((rows >= 0) & (rows < Nt))[:, None]
    at = rows.long().clamp(0, Nt - 1)
    codes, scales = four_bits.random(gen, Ng, Nk, Nc=Nc)
    xc, xs = four_bits.random(gen, Nt, Nc=Nc)
    x, d = _whole(gen, Nt, Nc), _whole(gen, Np, Nk)
    ker = four_bits.values(codes, scales, Nc)
    k, s, r = codes.cuda(), scales.cuda(), rows.cuda()
    calls = [(lambda t, o: routed.group_fwd4(x.cuda(), k, s, t, o, r), Nk, x.double()),
             (lambda t, o: routed.group_fwd4(xc.cuda(), k, s, t, o, r, InScales=xs.cuda()), Nk, four_bits.values(xc, xs, Nc)),
             (lambda t, o: routed.group_bwd_in4(d.cuda(), k, s, t, o), Nc, None)]
    bad = [offsets.clone() for _ in range(5)]
    bad[0][0] = 1
    bad[1][-1] = Np + 1
    bad[2][Ng // 2] = -5
    bad[3][Ng // 2], bad[3][-1] = Np, Np - 1
    bad[4][0], bad[4][-1] = -(1 << 31), (1 << 31) - 1
    for run, n, v in calls:
        for dtype in OUT.values():
            if v is not None:
                got = _out(Np, n, dtype)
                run(got, offsets.cuda())
                assert torch.equal(got.cpu(), _product(torch.where(there, v[at], 0.0), ker, offsets).to(dtype))
            for o in bad:
                got = _out(Np + 2, n, dtype)
                run(got[1:-1], o.cuda())
                assert torch.isnan(got).all()
