"""The routed contractions (router, grouped products, return, adapters) on the
GPU, against their definitions in 64 bits on the CPU.

Tolerances are bounds, not measurements: a sum of n products in fp32, in any
order, is off by at most (n + 8) 2^-24 of the sum of the products' magnitudes,
a bf16 result by 2^-8 of itself more (half a unit in the last place is 2^-9)."""
import math

import pytest
import torch

from gpu_helpers import say
from paper_2105_13480_amd import cnn, routed

pytestmark = pytest.mark.gpu

TYPES = {"f32": (torch.float32, torch.float32), "bf16": (torch.bfloat16, torch.float32),
         "bf16_obf16": (torch.bfloat16, torch.bfloat16)}
INF = math.inf


def _gpu(t):
    return t.cuda()


def _rand(gen, *shape, dtype=torch.float32):
    return torch.randn(shape, generator=gen).to(dtype)


def _at(t, shift):
    """The tensor on the GPU, `shift` elements past an aligned address."""
    flat = torch.empty(t.numel() + shift, dtype=t.dtype, device="cuda")
    flat[shift:] = t.reshape(-1).cuda()
    return flat[shift:].view(t.shape)


def _result(*shape, dtype=torch.float32):
    return torch.full(shape, math.nan, dtype=dtype, device="cuda")


def _close(got, want, mag, n, to):
    """want, mag: the exact result and the sum of its products' magnitudes."""
    got = got.double().cpu()
    tol = (n + 8) * 2.0 ** -24 * mag
    if to is torch.bfloat16:
        tol = tol + 2.0 ** -8 * (want.abs() + tol)
    bad = ~((got - want).abs() <= tol)
    assert not bad.any(), (f"{int(bad.sum())} of {bad.numel()} outside the bound, first at "
                           f"{torch.nonzero(bad)[0].tolist()}: {got[bad][0]} for {want[bad][0]}")


# ---- the grouped order ------------------------------------------------------

def _order(choice, Ng):
    """Offsets, rows and slots by counting, on the host."""
    Nt, Kt = choice.shape
    members = [[] for _ in range(Ng)]
    for t in range(Nt):
        for j in range(Kt):
            if choice[t, j] >= 0:
                members[int(choice[t, j])].append((t, j))
    offsets, rows = [0], []
    slots = torch.full((Nt, Kt), -1, dtype=torch.int32)
    for m in members:
        for t, j in m:
            slots[t, j] = len(rows)
            rows.append(t)
        offsets.append(len(rows))
    rows += [-1] * (Nt * Kt - len(rows))
    return (torch.tensor(offsets, dtype=torch.int32), torch.tensor(rows, dtype=torch.int32), slots)


def _choice(gen, Nt, Ng, Kt, active=None, drop=0.0):
    active = Ng if active is None else active
    used = torch.randperm(Ng, generator=gen)[:active]
    pick = torch.argsort(torch.rand((Nt, active), generator=gen), 1)[:, :Kt]
    choice = used[pick].int()
    choice[torch.rand(Nt, generator=gen) < drop] = -1
    return choice


# ---- router -----------------------------------------------------------------

def _route_oracle(logits, Kt, over):
    """Choice and weights row by row from the definition, in Python floats."""
    l = logits.double().tolist()
    choice, gates = [], []
    for row in l:
        allowed = [e for e, x in enumerate(row) if x > -INF]
        best = sorted(allowed, key=lambda e: (-row[e], e))[:Kt]
        top = row[best[0]] if best else 0.0
        w = lambda e: 1.0 if row[e] == top else math.exp(row[e] - top)  # noqa: E731
        total = sum(w(e) for e in (allowed if over == "all" else best))
        choice.append(best + [-1] * (Kt - len(best)))
        gates.append([w(e) / total for e in best] + [0.0] * (Kt - len(best)))
    return (torch.tensor(choice, dtype=torch.int32).reshape(len(l), Kt),
            torch.tensor(gates, dtype=torch.float64).reshape(len(l), Kt))


def _check_route(logits, Kt, over, shift=0):
    Nt, Ng = logits.shape
    r = routed.Routing(Nt, Ng, Kt)
    for t in (r.choice, r.offsets, r.rows, r.slots):
        t.fill_(-77)
    r.gates.fill_(math.nan)
    if r.ws is not None:
        r.ws.fill_(0xff)
    routed.route(_at(logits, shift), r, over=over)
    choice, gates = _route_oracle(logits, Kt, over)
    offsets, rows, slots = _order(choice, Ng)
    torch.cuda.synchronize()
    assert torch.equal(r.choice.cpu(), choice)
    assert torch.equal(r.offsets.cpu(), offsets)
    assert torch.equal(r.rows.cpu(), rows)
    assert torch.equal(r.slots.cpu(), slots)
    # exp to a few units, a sum of at most Ng terms, one division
    tol = (Ng + 16) * 2.0 ** -24
    assert ((r.gates.double().cpu() - gates).abs() <= tol * gates + 1e-38).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("over", ["all", "chosen"])
@pytest.mark.parametrize("Nt,Ng,Kt", [(1, 1, 1), (1, 4, 4), (3, 7, 2), (64, 32, 4), (65, 33, 5),
                                      (100, 64, 8), (517, 130, 8), (130, 256, 16), (67, 257, 3),
                                      (66, 1024, 16), (4100, 16, 2)])
def test_route(Nt, Ng, Kt, over, dtype):
    say(f"[route] {Nt} {Ng} {Kt} {over} {dtype}")
    gen = torch.Generator().manual_seed(Nt * 31 + Ng)
    logits = (torch.randn((Nt, Ng), generator=gen) * 2).to(dtype)
    # bf16 logits tie by themselves; fp32 ones are made to
    logits = torch.where(torch.rand((Nt, Ng), generator=gen) < 0.3, logits[:, :1], logits)
    _check_route(logits, Kt, over, shift=Nt % 2)


@pytest.mark.parametrize("over", ["all", "chosen"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_route_masks(dtype, over):
    """Rows barred from some or all experts, lowest values, infinities, NaN, zeros of both signs."""
    say(f"[route] masks {over} {dtype}")
    low = torch.finfo(dtype).min
    rows = [[-INF] * 6, [-INF, 1.0, -INF, -INF, -INF, -INF], [low] * 6, [low, -INF, low, 0.0, low, -INF],
            [math.nan] * 6, [math.nan, 2.0, math.nan, -3.0, 2.0, 1.0], [INF, 0.0, INF, 1.0, -INF, 2.0],
            [-0.0, 0.0, -0.0, 0.0, -1.0, 1.0], [1e38, -1e38, 3e38, -3e38, 0.0, 1.0],
            [-80.0, 20.0, -200.0, 20.0, 19.0, -1e4]]
    logits = torch.tensor(rows * 9, dtype=torch.float32).to(dtype)
    for Kt in (1, 3, 6):
        _check_route(logits, Kt, over)


def test_route_no_rows():
    r = routed.Routing(0, 8, 2)
    r.offsets.fill_(5)
    routed.route(torch.empty((0, 8), device="cuda"), r)
    assert r.offsets.tolist() == [0] * 9


@pytest.mark.parametrize("mode", TYPES)
@pytest.mark.parametrize("over", ["all", "chosen"])
@pytest.mark.parametrize("Nt,Ng,Kt", [(1, 1, 1), (5, 3, 2), (33, 64, 4), (40, 200, 8), (17, 700, 16)])
def test_route_bwd(Nt, Ng, Kt, over, mode):
    say(f"[route_bwd] {Nt} {Ng} {Kt} {over} {mode}")
    ti, to = TYPES[mode]
    gen = torch.Generator().manual_seed(Nt + Ng)
    logits = _rand(gen, Nt, Ng, dtype=ti)
    logits[torch.rand((Nt, Ng), generator=gen) < 0.2] = -INF
    if Nt > 4:
        logits[2] = -INF
    choice, gates = _route_oracle(logits, Kt, over)
    dg = _rand(gen, Nt, Kt)
    out = _result(Nt, Ng, dtype=to)
    routed.route_bwd(_gpu(logits), _gpu(choice), _gpu(gates.float()), _gpu(dg), out, over=over)
    # autograd of the definition in 64 bits
    x = logits.double().requires_grad_()
    loss = torch.zeros((), dtype=torch.float64)
    for t in range(Nt):
        best = [int(e) for e in choice[t] if e >= 0]
        if best:
            pool = [e for e in range(Ng) if logits[t, e] > -INF] if over == "all" else best
            p = torch.softmax(x[t, pool], 0)
            for j, e in enumerate(best):
                loss = loss + p[pool.index(e)] * dg[t, j].double()
    if loss.requires_grad:
        loss.backward()
    want = x.grad if x.grad is not None else torch.zeros_like(x)
    want = torch.nan_to_num(want)
    mag = dg.double().abs().sum(1, keepdim=True).expand(Nt, Ng) * 2
    _close(out, want, mag, Ng + Kt + 16, to)


def test_route_bwd_differences():
    """The gradient against differences of the forward pass itself."""
    gen = torch.Generator().manual_seed(3)
    logits, dg = _rand(gen, 1, 8), _rand(gen, 1, 3)
    for over in ("all", "chosen"):
        r = routed.route(_gpu(logits), routed.Routing(1, 8, 3), over=over)
        d = _result(1, 8)
        routed.route_bwd(_gpu(logits), r.choice, r.gates, _gpu(dg), d, over=over)
        for e in range(8):
            h = 2.0 ** -8
            f = []
            for s in (h, -h):
                moved = logits.clone()
                moved[0, e] += s
                q = routed.route(_gpu(moved), routed.Routing(1, 8, 3), over=over)
                assert torch.equal(q.choice, r.choice)
                f.append(float((q.gates.cpu().double() * dg.double()).sum()))
            # third derivative of a softmax below 1 a weight: h^2 / 6; fp32 weights: 2^-22 / h
            assert abs((f[0] - f[1]) / (2 * h) - float(d[0, e])) < float(dg.abs().sum()) * (h * h + 2.0 ** -22 / h)


# ---- return -----------------------------------------------------------------

COMBINE = [(1, 1, 1, 1), (1, 4, 2, 8), (7, 5, 3, 65), (33, 16, 4, 256), (20, 8, 8, 517), (3, 64, 16, 2048),
           (300, 8, 2, 12)]


@pytest.mark.parametrize("mode", TYPES)
@pytest.mark.parametrize("Nt,Ng,Kt,Nk", COMBINE)
@pytest.mark.parametrize("weighted", [True, False])
def test_combine(Nt, Ng, Kt, Nk, weighted, mode):
    say(f"[combine] {Nt} {Ng} {Kt} {Nk} {weighted} {mode}")
    ti, to = TYPES[mode]
    gen = torch.Generator().manual_seed(Nt * 7 + Nk)
    Kt = min(Kt, Ng)
    choice = _choice(gen, Nt, Ng, Kt, drop=0.2 if Nt > 5 else 0.0)
    offsets, rows, slots = _order(choice, Ng)
    In = _rand(gen, Nt * Kt, Nk, dtype=ti)
    In[int(offsets[-1]):] = math.nan  # no pair's rows are not read
    gates = torch.rand((Nt, Kt), generator=gen)
    out = _result(Nt, Nk, dtype=to)
    routed.combine(_at(In, Nk % 2), out, _gpu(slots), _gpu(gates) if weighted else None)
    want = torch.zeros((Nt, Nk), dtype=torch.float64)
    mag = want.clone()
    for t in range(Nt):
        for j in range(Kt):
            if slots[t, j] >= 0:
                v = In[slots[t, j]].double() * (gates[t, j].double() if weighted else 1.0)
                want[t] += v
                mag[t] += v.abs()
    _close(out, want, mag, Kt, to)


@pytest.mark.parametrize("mode", TYPES)
@pytest.mark.parametrize("Nt,Ng,Kt,Nk", COMBINE)
@pytest.mark.parametrize("weighted", [True, False])
def test_combine_bwd(Nt, Ng, Kt, Nk, weighted, mode):
    say(f"[combine_bwd] {Nt} {Ng} {Kt} {Nk} {weighted} {mode}")
    ti, to = TYPES[mode]
    gen = torch.Generator().manual_seed(Nt * 5 + Nk)
    Kt = min(Kt, Ng)
    choice = _choice(gen, Nt, Ng, Kt, drop=0.2 if Nt > 5 else 0.0)
    offsets, rows, slots = _order(choice, Ng)
    Np = Nt * Kt
    In, dOut = _rand(gen, Np, Nk, dtype=ti), _rand(gen, Nt, Nk, dtype=ti)
    gates = torch.rand((Nt, Kt), generator=gen)
    dIn, dG = _result(Np, Nk, dtype=to), _result(Nt, Kt)
    routed.combine_bwd(_gpu(dOut), _at(In, 1), dIn, dG, _gpu(slots), _gpu(rows),
                       _gpu(gates) if weighted else None)
    wi, wg, mg = (torch.zeros(s, dtype=torch.float64) for s in ((Np, Nk), (Nt, Kt), (Nt, Kt)))
    for t in range(Nt):
        for j in range(Kt):
            p = int(slots[t, j])
            if p >= 0:
                wi[p] = dOut[t].double() * (gates[t, j].double() if weighted else 1.0)
                prod = dOut[t].double() * In[p].double()
                wg[t, j], mg[t, j] = prod.sum(), prod.abs().sum()
    _close(dIn, wi, wi.abs(), 1, to)
    _close(dG, wg, mg, Nk, torch.float32)


# ---- grouped products -------------------------------------------------------

# (Nt, Ng, active, Kt, drop, Nc, Nk): single rows, few rows a group (straight from
# memory), whole tiles, ragged and odd extents, idle groups, rows without a group
GROUP = [(1, 1, 1, 1, 0.0, 1, 1), (1, 4, 2, 1, 0.0, 64, 32), (2, 3, 3, 2, 0.0, 130, 33),
         (5, 8, 6, 2, 0.0, 256, 128), (9, 2, 2, 1, 0.3, 2048, 48), (16, 4, 3, 2, 0.2, 520, 100),
         (40, 3, 2, 1, 0.0, 96, 80), (70, 2, 2, 2, 0.1, 72, 136), (200, 3, 2, 2, 0.2, 136, 264),
         (300, 2, 2, 1, 0.0, 515, 131), (257, 1, 1, 1, 0.0, 64, 129), (500, 70, 66, 2, 0.1, 40, 24),
         (600, 2, 1, 1, 0.5, 200, 640), (1100, 2, 2, 1, 0.1, 192, 328), (700, 1, 1, 1, 0.0, 1000, 520)]


def _group_data(case, mode, seed):
    Nt, Ng, active, Kt, drop, Nc, Nk = case
    ti, _ = TYPES[mode]
    gen = torch.Generator().manual_seed(seed)
    choice = _choice(gen, Nt, Ng, Kt, active, drop)
    offsets, rows, _ = _order(choice, Ng)
    return (offsets, rows, _rand(gen, Nt, Nc, dtype=ti), _rand(gen, Ng, Nk, Nc, dtype=ti),
            _rand(gen, Nt * Kt, Nk, dtype=ti))


@pytest.mark.parametrize("mode", TYPES)
@pytest.mark.parametrize("case", GROUP, ids=str)
@pytest.mark.parametrize("gathered", [True, False])
def test_group_fwd(case, gathered, mode):
    say(f"[group_fwd] {case} {gathered} {mode}")
    _, to = TYPES[mode]
    offsets, rows, In, Ker, _ = _group_data(case, mode, 11)
    Ng, Nk, Nc = Ker.shape
    Np = rows.numel()
    x = In[rows.long().clamp_min(0)]
    shift = 1 if case[0] == 300 else 0
    out = _result(Np + 1, Nk, dtype=to)
    if gathered:
        routed.group_fwd(_at(In, shift), _at(Ker, shift), out[:Np], _gpu(offsets), _gpu(rows))
    else:
        routed.group_fwd(_at(x, shift), _at(Ker, shift), out[:Np], _gpu(offsets))
    want = torch.zeros((Np, Nk), dtype=torch.float64)
    mag = want.clone()
    for g in range(Ng):
        lo, hi = int(offsets[g]), int(offsets[g + 1])
        want[lo:hi] = x[lo:hi].double() @ Ker[g].double().t()
        mag[lo:hi] = x[lo:hi].double().abs() @ Ker[g].double().abs().t()
    _close(out[:Np], want, mag, Nc, to)
    assert torch.isnan(out[Np]).all()


@pytest.mark.parametrize("mode", TYPES)
@pytest.mark.parametrize("case", GROUP, ids=str)
def test_group_bwd_in(case, mode):
    say(f"[group_bwd_in] {case} {mode}")
    _, to = TYPES[mode]
    offsets, rows, _, Ker, dOut = _group_data(case, mode, 12)
    Ng, Nk, Nc = Ker.shape
    Np = rows.numel()
    shift = 1 if case[0] == 300 else 0
    out = _result(Np + 1, Nc, dtype=to)
    routed.group_bwd_in(_at(dOut, shift), _at(Ker, shift), out[:Np], _gpu(offsets))
    want = torch.zeros((Np, Nc), dtype=torch.float64)
    mag = want.clone()
    for g in range(Ng):
        lo, hi = int(offsets[g]), int(offsets[g + 1])
        want[lo:hi] = dOut[lo:hi].double() @ Ker[g].double()
        mag[lo:hi] = dOut[lo:hi].double().abs() @ Ker[g].double().abs()
    _close(out[:Np], want, mag, Nk, to)
    assert torch.isnan(out[Np]).all()


@pytest.mark.parametrize("mode", TYPES)
@pytest.mark.parametrize("case", GROUP, ids=str)
@pytest.mark.parametrize("gathered", [True, False])
def test_group_bwd_ker(case, gathered, mode):
    say(f"[group_bwd_ker] {case} {gathered} {mode}")
    _, to = TYPES[mode]
    offsets, rows, In, Ker, dOut = _group_data(case, mode, 13)
    Ng, Nk, Nc = Ker.shape
    x = In[rows.long().clamp_min(0)]
    P = int(offsets[-1])
    dOut[P:] = math.nan  # rows without a group take no part
    if not gathered:
        x[P:] = math.nan
    shift = 1 if case[0] == 300 else 0
    out = _result(Ng + 1, Nk, Nc, dtype=to)
    if gathered:
        routed.group_bwd_ker(_at(dOut, shift), _at(In, shift), out[:Ng], _gpu(offsets), _gpu(rows))
    else:
        routed.group_bwd_ker(_at(dOut, shift), _at(x, shift), out[:Ng], _gpu(offsets))
    n = int((offsets[1:] - offsets[:-1]).max())
    want = torch.zeros((Ng, Nk, Nc), dtype=torch.float64)
    mag = want.clone()
    for g in range(Ng):
        lo, hi = int(offsets[g]), int(offsets[g + 1])
        want[g] = dOut[lo:hi].double().t() @ x[lo:hi].double()
        mag[g] = dOut[lo:hi].double().abs().t() @ x[lo:hi].double().abs()
    _close(out[:Ng], want, mag, n, to)
    assert torch.isnan(out[Ng]).all()


def test_group_rows_outside_read_as_zeros():
    """Row indices outside the source are zero rows, in every product and on every path."""
    gen = torch.Generator().manual_seed(4)
    for n, Nc in ((3, 64), (3, 63), (200, 64), (200, 63)):
        In, Ker = _rand(gen, 5, Nc), _rand(gen, 1, 16, Nc)
        rows = torch.randint(0, 5, (n,), generator=gen).int()
        rows[1], rows[2] = 5, -9
        off = torch.tensor([0, n], dtype=torch.int32)
        out = _result(n, 16)
        routed.group_fwd(_gpu(In), _gpu(Ker), out, _gpu(off), _gpu(rows))
        assert (out[1:3] == 0).all() and (out[0] != 0).any()
        d = torch.zeros((n, 16))
        d[1:3] = 1.0
        dk = _result(1, 16, Nc)
        routed.group_bwd_ker(_gpu(d), _gpu(In), dk, _gpu(off), _gpu(rows))
        assert (dk == 0).all()


def test_group_values_stay_in_their_rows():
    """NaN and infinities in one row or group leave the others' results alone."""
    gen = torch.Generator().manual_seed(5)
    for mode in TYPES:
        ti, to = TYPES[mode]
        for n, Nc in ((6, 64), (300, 72), (300, 67)):
            In, Ker = _rand(gen, n, Nc, dtype=ti), _rand(gen, 3, 40, Nc, dtype=ti)
            off = torch.tensor([0, n // 2, n // 2 + 1, n - 1], dtype=torch.int32)
            clean, dirty = _result(n, 40, dtype=to), _result(n, 40, dtype=to)
            routed.group_fwd(_gpu(In), _gpu(Ker), clean, _gpu(off))
            In[0, 0], In[n // 2] = INF, math.nan
            Ker[1] = math.nan
            In[n - 1] = math.nan  # no group
            routed.group_fwd(_gpu(In), _gpu(Ker), dirty, _gpu(off))
            keep = torch.ones(n, dtype=torch.bool)
            keep[[0, n // 2]] = False
            assert torch.equal(clean[keep.cuda()], dirty[keep.cuda()])
            assert not torch.isfinite(dirty[[0, n // 2]].float()).any()
            dk = _result(3, 40, Nc, dtype=to)
            routed.group_bwd_ker(_gpu(_rand(gen, n, 40, dtype=ti)), _gpu(In), dk, _gpu(off))
            assert torch.isfinite(dk[2].float()).all() and torch.isnan(dk[1].float()).all()


def test_group_no_rows():
    Ker = torch.ones((3, 8, 16), device="cuda")
    off = torch.zeros(4, dtype=torch.int32, device="cuda")
    none = torch.empty((0, 16), device="cuda")
    assert routed.group_fwd(none, Ker, torch.empty((0, 8), device="cuda"), off).shape == (0, 8)
    dk = routed.group_bwd_ker(torch.empty((0, 8), device="cuda"), none, _result(3, 8, 16), off)
    assert (dk == 0).all()
    # rows, none of which has a group
    out = routed.group_fwd(torch.ones((40, 16), device="cuda"), Ker, _result(40, 8), off)
    assert (out == 0).all()
    din = routed.group_bwd_in(torch.ones((40, 8), device="cuda"), Ker, _result(40, 16), off)
    assert (din == 0).all()


def test_rows_beyond_32_bits():
    """Rows whose first element lies past 2^31 elements (and 2^32 bytes)."""
    gen = torch.Generator().manual_seed(7)
    Nt, Nc, Nk = (1 << 31) // 2048 + 300, 2048, 24
    In = torch.empty((Nt, Nc), dtype=torch.bfloat16, device="cuda")
    Ker = _rand(gen, 2, Nk, Nc, dtype=torch.bfloat16)
    for n in (5, 200):
        rows = torch.cat([torch.tensor([0, Nt - 1]), torch.randint(Nt - 290, Nt, (n - 2,), generator=gen)])
        x = _rand(gen, n, Nc, dtype=torch.bfloat16)
        where = {int(r): i for i, r in enumerate(rows)}  # the last of equal rows
        for r, i in where.items():
            In[r] = x[i].cuda()
        x = x[[where[int(r)] for r in rows]]
        off = torch.tensor([0, n // 2, n], dtype=torch.int32)
        out = _result(n, Nk)
        routed.group_fwd(In, _gpu(Ker), out, _gpu(off), _gpu(rows.int()))
        k = [Ker[0 if p < n // 2 else 1] for p in range(n)]
        want = torch.stack([k[p].double() @ x[p].double() for p in range(n)])
        mag = torch.stack([k[p].double().abs() @ x[p].double().abs() for p in range(n)])
        _close(out, want, mag, Nc, torch.float32)


# ---- adapters ---------------------------------------------------------------

# (Nt, Nc, Nk, Na, Nl, run): few rows (as they come) and many (in order), ranks
# below, at and above a unit, one row, odd extents, runs of one and many rows
ADAPT = [(1, 1, 1, 1, 1, 1), (1, 64, 48, 3, 8, 1), (3, 70, 33, 2, 3, 1), (16, 2048, 64, 5, 16, 2),
         (40, 515, 100, 9, 12, 3), (64, 4096, 40, 40, 64, 1), (64, 256, 128, 2, 33, 20), (65, 128, 64, 3, 8, 10),
         (130, 136, 200, 1, 16, 130), (200, 72, 136, 70, 4, 1), (333, 201, 157, 5, 12, 30),
         (513, 256, 520, 4, 64, 100), (700, 64, 64, 3, 130, 50)]


@pytest.mark.parametrize("mode", TYPES)
@pytest.mark.parametrize("case", ADAPT, ids=str)
@pytest.mark.parametrize("scaled", [True, False])
def test_adapt(case, scaled, mode):
    say(f"[adapt] {case} {scaled} {mode}")
    Nt, Nc, Nk, Na, Nl, run = case
    ti, to = TYPES[mode]
    gen = torch.Generator().manual_seed(Nt + Nl)
    In, Ker = _rand(gen, Nt, Nc, dtype=ti), _rand(gen, Nk, Nc, dtype=ti)
    A, B = _rand(gen, Na, Nl, Nc, dtype=ti), _rand(gen, Na, Nk, Nl, dtype=ti)
    ids = torch.randint(-1, Na + 1, (Nt,), generator=gen)[torch.arange(Nt) // run].int()  # Na: none, too
    scales = torch.rand(Na, generator=gen) + 0.5
    out = _result(Nt + 1, Nk, dtype=to)
    shift = Nt % 2
    gin, gk, ga, gb = (_at(t, shift) for t in (In, Ker, A, B))
    ws = routed.adapt_workspace(gin, gk, ga, out[:Nt])
    ws.fill_(0xff)
    routed.adapt_fwd(gin, gk, ga, gb, _gpu(ids), out[:Nt], _gpu(scales) if scaled else None, ws)
    x = In.double()
    want, mag = x @ Ker.double().t(), x.abs() @ Ker.double().abs().t()
    for a in range(Na):
        t = torch.nonzero(ids == a).reshape(-1)
        s = float(scales[a]) if scaled else 1.0
        want[t] += s * ((x[t] @ A[a].double().t()) @ B[a].double().t())
        mag[t] += s * ((x[t].abs() @ A[a].double().abs().t()) @ B[a].double().abs().t())
    # both sums, the scale, and (bf16 result) H kept to 2^-15 of itself
    n = 2 * Nc + Nl + (2 ** 9 if to is torch.bfloat16 else 0)
    _close(out[:Nt], want, mag, n, to)
    assert torch.isnan(out[Nt].float()).all()


def test_adapt_values_stay_in_their_rows():
    """An adapter with infinities or NaN reaches only the rows that name it."""
    gen = torch.Generator().manual_seed(6)
    for mode in TYPES:
        ti, to = TYPES[mode]
        for Nt in (30, 200):
            In, Ker = _rand(gen, Nt, 72, dtype=ti), _rand(gen, 40, 72, dtype=ti)
            A, B = _rand(gen, 3, 8, 72, dtype=ti), _rand(gen, 3, 40, 8, dtype=ti)
            ids = torch.randint(-1, 3, (Nt,), generator=gen).int()
            res = []
            for dirty in (False, True):
                if dirty:
                    A[1, 2], B[1, 5] = INF, math.nan
                out = _result(Nt, 40, dtype=to)
                routed.adapt_fwd(_gpu(In), _gpu(Ker), _gpu(A), _gpu(B), _gpu(ids), out, None,
                                 routed.adapt_workspace(_gpu(In), Ker, A, out))
                res.append(out.float().cpu())
            other = ids != 1
            assert torch.equal(res[0][other], res[1][other])
            assert not torch.isfinite(res[1][~other]).any()


# ---- use --------------------------------------------------------------------

def test_other_stream_and_graph():
    """Calls on a stream of the caller's, and a graph of a whole routed layer
    replayed on new inputs: every replay equals the plain calls."""
    gen = torch.Generator().manual_seed(8)
    Nt, Ng, Kt, Nc, Nk = 300, 6, 2, 64, 72
    Ker = _gpu(_rand(gen, Ng, Nk, Nc, dtype=torch.bfloat16))
    logits, In = torch.empty((Nt, Ng), device="cuda"), torch.empty((Nt, Nc), dtype=torch.bfloat16, device="cuda")
    r = routed.Routing(Nt, Ng, Kt)
    mid, out = _result(Nt * Kt, Nk, dtype=torch.bfloat16), _result(Nt, Nk)

    def layer():
        routed.route(logits, r)
        routed.group_fwd(In, Ker, mid, r.offsets, r.rows)
        routed.combine(mid, out, r.slots, r.gates)

    data = [(_rand(gen, Nt, Ng), _rand(gen, Nt, Nc, dtype=torch.bfloat16)) for _ in range(3)]
    want = []
    for l, x in data:
        logits.copy_(l), In.copy_(x)
        layer()
        want.append(out.clone())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer()
    side.synchronize()
    assert torch.equal(out, want[-1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer()
    for i in (0, 1, 2, 1, 0):
        logits.copy_(data[i][0]), In.copy_(data[i][1])
        out.fill_(math.nan)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[i])


def test_repeats_bit_for_bit():
    gen = torch.Generator().manual_seed(9)
    x, k = _gpu(_rand(gen, 500, 520)), _gpu(_rand(gen, 4, 264, 520))
    off = torch.tensor([0, 100, 100, 430, 480], dtype=torch.int32, device="cuda")
    first = routed.group_fwd(x, k, _result(500, 264), off)
    for _ in range(3):
        assert torch.equal(first, routed.group_fwd(x, k, _result(500, 264), off))


def test_refusals():
    """The binding's own checks (the library's are tested without a GPU)."""
    x, k = torch.zeros((8, 16), device="cuda"), torch.zeros((2, 4, 16), device="cuda")
    off, out = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros((8, 4), device="cuda")
    bad = [lambda: routed.group_fwd(x.cpu(), k, out, off), lambda: routed.group_fwd(x.t(), k, out, off),
           lambda: routed.group_fwd(x, k, out[:7], off), lambda: routed.group_fwd(x, k, out, off.long()),
           lambda: routed.group_fwd(x, k, out, off[:2]), lambda: routed.group_fwd(x.bfloat16(), k, out, off),
           lambda: routed.group_fwd(x, k, out.bfloat16(), off), lambda: routed.group_fwd(x.double(), k.double(), out, off),
           lambda: routed.group_fwd(x, k, out, off, off), lambda: routed.group_bwd_in(out, k, x[:, :8], off),
           lambda: routed.group_bwd_ker(out, x, k[:, :2], off),
           lambda: routed.route(x, routed.Routing(8, 15, 2)), lambda: routed.route(x, routed.Routing(8, 16, 2), over="some"),
           lambda: routed.combine(out, x, off.view(3, 1))]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    with pytest.raises(cnn.CnnError) as e:
        routed.group_fwd(x, k, x.view(-1)[:32].view(8, 4), off)
    assert e.value.status == -5
    with pytest.raises(cnn.CnnError) as e:
        routed.Routing(8, 4, 5)
    assert e.value.status == -2
    with pytest.raises(cnn.CnnError) as e:  # a workspace too small
        a, b = torch.zeros((1, 4, 16), device="cuda"), torch.zeros((1, 4, 4), device="cuda")
        routed.adapt_fwd(x, k[0], a, b, off[:1].expand(8).contiguous(), out, None,
                         torch.empty(8, dtype=torch.uint8, device="cuda"))
    assert e.value.status == -2
