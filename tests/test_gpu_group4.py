"""Grouped products with Ker (and rows) in 4 bits, against the definition in 64
bits on the CPU.

With scales near one and whole numbers no sum leaves fp32, so results are exact.
Otherwise: a sum of n products in fp32, in any order, is off by at most (n + 8)
2^-24 of the sum of the products' magnitudes, a bf16 result by 2^-8 of itself
more."""
import math

import pytest
import torch

import four_bits
from gpu_helpers import say
from paper_2105_13480_amd import cnn, routed

pytestmark = pytest.mark.gpu

OUT = {"f32": torch.float32, "bf16": torch.bfloat16}

# (Nt, Ng, active, Kt, drop, Nc, Nk): one row and one value, few rows a group, whole and
# ragged tiles of each size, last rounds that are halved, rows that end inside a block, idle groups, more than 64 of
# them, rows without a group
CASES = [(1, 1, 1, 1, 0.0, 1, 1), (1, 4, 2, 1, 0.0, 64, 32), (2, 3, 3, 2, 0.0, 130, 33),
         (5, 8, 6, 2, 0.0, 256, 128), (9, 2, 2, 1, 0.3, 2048, 48), (16, 4, 3, 2, 0.2, 520, 100),
         (8, 32, 20, 4, 0.0, 1024, 80), (40, 3, 2, 1, 0.0, 96, 80), (70, 2, 2, 2, 0.1, 72, 136),
         (100, 9, 7, 2, 0.0, 1600, 272), (200, 3, 2, 2, 0.2, 136, 264), (300, 2, 2, 1, 0.0, 515, 131),
         (257, 1, 1, 1, 0.0, 64, 129), (500, 70, 66, 2, 0.1, 40, 24), (600, 2, 1, 1, 0.5, 200, 640),
         (1100, 2, 2, 1, 0.1, 192, 328), (700, 1, 1, 1, 0.0, 1000, 520), (333, 12, 11, 2, 0.0, 1001, 537),
         (640, 28, 26, 1, 0.0, 1056, 2048), (1300, 3, 3, 2, 0.1, 1152, 2112), (2600, 2, 2, 2, 0.05, 640, 3000),
         (3000, 1, 1, 1, 0.0, 1280, 2304), (4100, 5, 5, 1, 0.02, 2304, 1290), (20, 2, 2, 1, 0.0, 3008, 250),
         (6001, 1, 1, 1, 0.0, 267, 2071), (4800, 16, 15, 1, 0.1, 1536, 1544), (8000, 5, 5, 1, 0.05, 1000, 2056),
         (400, 40, 30, 1, 0.0, 2112, 500), (5000, 3, 3, 1, 0.05, 2056, 2056),
         (8200, 3, 3, 1, 0.05, 2304, 2056), (8000, 2, 2, 1, 0.02, 2056, 1544)]


def _order(gen, Nt, Ng, active, Kt, drop):
    """Offsets and rows by counting."""
    used = torch.randperm(Ng, generator=gen)[:active]
    pick = used[torch.argsort(torch.rand((Nt, active), generator=gen), 1)[:, :Kt]]
    pick[torch.rand(Nt, generator=gen) < drop] = -1
    offsets, rows = [0], []
    for g in range(Ng):
        rows += torch.nonzero((pick == g).any(1)).reshape(-1).tolist()
        offsets.append(len(rows))
    rows += [-1] * (Nt * pick.shape[1] - len(rows))
    return torch.tensor(offsets, dtype=torch.int32), torch.tensor(rows, dtype=torch.int32)


def _whole(gen, *shape, top=3):
    return torch.randint(-top, top + 1, shape, generator=gen).bfloat16()


def _at(t, shift):
    flat = torch.empty(t.numel() + shift, dtype=t.dtype, device="cuda")
    flat[shift:] = t.reshape(-1).cuda()
    return flat[shift:].view(t.shape)


def _out(n, m, dtype):
    return torch.full((n, m), math.nan, dtype=dtype, device="cuda")


def _product(x, ker, offsets):
    """x [Np, K] by ker [Ng, M, K], group by group; zeros past the last."""
    want = torch.zeros((x.shape[0], ker.shape[1]), dtype=x.dtype)
    for g in range(ker.shape[0]):
        lo, hi = int(offsets[g]), int(offsets[g + 1])
        want[lo:hi] = x[lo:hi] @ ker[g].t()
    return want


@pytest.mark.parametrize("out", OUT)
@pytest.mark.parametrize("case", CASES, ids=str)
@pytest.mark.parametrize("both", [False, True])
def test_forward(case, both, out):
    """Gathered rows and rows in order; bf16 rows at an odd element, scales at an odd
    byte or not."""
    say(f"[fwd4] {case} {both} {out}")
    Nt, Ng, active, Kt, drop, Nc, Nk = case
    gen = torch.Generator().manual_seed(Nt + Nc)
    offsets, rows = _order(gen, Nt, Ng, active, Kt, drop)
    codes, scales = four_bits.random(gen, Ng, Nk, Nc=Nc)
    if both:
        xc, xs = four_bits.random(gen, Nt, Nc=Nc)
        x = four_bits.values(xc, xs, Nc)
    else:
        x = _whole(gen, Nt, Nc).double()
    p = x[rows.long().clamp_min(0)]
    want = _product(p, four_bits.values(codes, scales, Nc), offsets)
    Np = rows.numel()
    for gathered in (True, False):
        got = _out(Np + 1, Nk, OUT[out])
        at = rows.long().clamp_min(0)
        if both:
            In, extra = (xc if gathered else xc[at]).cuda(), {"InScales": _at(xs if gathered else xs[at], int(Nt % 4 > 0))}
        else:
            In, extra = _at((x if gathered else p).bfloat16(), Nt % 2), {}
        routed.group_fwd4(In, codes.cuda(), _at(scales, int(Nt % 4 > 0)), got[:Np], offsets.cuda(),
                          rows.cuda() if gathered else None, **extra)
        assert torch.equal(got[:Np].cpu(), want.to(OUT[out]))
        assert torch.isnan(got[Np]).all()


@pytest.mark.parametrize("out", OUT)
@pytest.mark.parametrize("case", CASES, ids=str)
def test_gradient(case, out):
    say(f"[bwd4] {case} {out}")
    Nt, Ng, active, Kt, drop, Nc, Nk = case
    gen = torch.Generator().manual_seed(Nt + Nk)
    offsets, rows = _order(gen, Nt, Ng, active, Kt, drop)
    Np = rows.numel()
    codes, scales = four_bits.random(gen, Ng, Nk, Nc=Nc)
    d = _whole(gen, Np, Nk)
    want = _product(d.double(), four_bits.values(codes, scales, Nc).transpose(1, 2).contiguous(), offsets)
    got = _out(Np + 1, Nc, OUT[out])
    routed.group_bwd_in4(_at(d, Nt % 2), codes.cuda(), _at(scales, 1), got[:Np], offsets.cuda())
    assert torch.equal(got[:Np].cpu(), want.to(OUT[out]))
    assert torch.isnan(got[Np]).all()


@pytest.mark.parametrize("out", OUT)
@pytest.mark.parametrize("Nt,Nc,Nk,spread", [(5, 256, 128, 8), (300, 515, 131, 8), (40, 96, 80, 60), (1100, 1152, 520, 20)])
def test_values(Nt, Nc, Nk, spread, out):
    """Scales that differ widely, within the bound of an fp32 sum."""
    say(f"[values4] {Nt} {Nc} {Nk} {spread} {out}")
    gen = torch.Generator().manual_seed(Nt)
    Ng = 3
    offsets, rows = _order(gen, Nt, Ng, Ng, 2, 0.1)
    Np = rows.numel()
    codes, scales = four_bits.random(gen, Ng, Nk, Nc=Nc, low=127 - spread, high=128 + spread)
    ker = four_bits.values(codes, scales, Nc)
    xc, xs = four_bits.random(gen, Nt, Nc=Nc, low=127 - spread, high=128 + spread)
    x, d = torch.randn((Nt, Nc), generator=gen).bfloat16(), torch.randn((Np, Nk), generator=gen).bfloat16()
    at = rows.long().clamp_min(0)
    turned = ker.transpose(1, 2).contiguous()
    k, s, o, r = codes.cuda(), scales.cuda(), offsets.cuda(), rows.cuda()
    runs = [(x.double()[at], ker, lambda: routed.group_fwd4(x.cuda(), k, s, _out(Np, Nk, OUT[out]), o, r)),
            (four_bits.values(xc, xs, Nc)[at], ker,
             lambda: routed.group_fwd4(xc.cuda(), k, s, _out(Np, Nk, OUT[out]), o, r, InScales=xs.cuda())),
            (d.double(), turned, lambda: routed.group_bwd_in4(d.cuda(), k, s, _out(Np, Nc, OUT[out]), o))]
    for v, w, run in runs:
        want, mag = _product(v, w, offsets), _product(v.abs(), w.abs(), offsets)
        tol = (v.shape[1] + 8) * 2.0 ** -24 * mag
        if out == "bf16":
            tol = tol + 2.0 ** -8 * (want.abs() + tol)
        assert ((run().double().cpu() - want).abs() <= tol).all()


@pytest.mark.parametrize("Nt,Nc,Nk", [(1, 64, 8), (9, 96, 40), (100, 515, 72), (1500, 256, 300)])
def test_gradient_differences(Nt, Nc, Nk):
    """The forward product is linear in In: with whole numbers a difference over any
    step equals the gradient along it exactly."""
    say(f"[differences4] {Nt} {Nc} {Nk}")
    gen = torch.Generator().manual_seed(Nc)
    offsets, _ = _order(gen, Nt, 3, 3, 1, 0.0)
    codes, scales = four_bits.random(gen, 3, Nk, Nc=Nc)
    x, v, d = _whole(gen, Nt, Nc), _whole(gen, Nt, Nc, top=1), _whole(gen, Nt, Nk)
    k, s, o = codes.cuda(), scales.cuda(), offsets.cuda()
    f = lambda t: float((routed.group_fwd4(t.cuda(), k, s, _out(Nt, Nk, torch.float32), o).double().cpu() * d.double()).sum())  # noqa: E731
    g = routed.group_bwd_in4(d.cuda(), k, s, _out(Nt, Nc, torch.float32), o)
    assert f(x + v) - f(x - v) == 2 * float((g.double().cpu() * v.double()).sum())


@pytest.mark.parametrize("Nc,Nk", [(520, 136), (2048, 2048)])
@pytest.mark.parametrize("sizes", [[3, 1, 0, 5, 2], [40, 9, 0, 33, 7], [1300, 57, 0, 901, 2400]], ids=str)
def test_no_numbers_stay(sizes, Nc, Nk):
    """A NaN block, infinite scales and rows of NaN and infinities stay in their
    group, feature and row; places past the last group are zeros whatever they hold."""
    say(f"[isolation4] {sizes} {Nc} {Nk}")
    gen = torch.Generator(device="cuda").manual_seed(3)
    Ng, P = len(sizes), sum(sizes)
    Np = P + 7
    off = torch.tensor([0] + sizes).cumsum(0).int().cuda()
    x = torch.randn((Np, Nc), generator=gen, device="cuda").bfloat16()
    d = torch.randn((Np, Nk), generator=gen, device="cuda").bfloat16()
    w = torch.randn((Ng, Nk, Nc), generator=gen, device="cuda")
    Nb = four_bits.blocks(Nc)
    new = lambda *s: torch.empty(s, dtype=torch.uint8, device="cuda")  # noqa: E731
    k, s = routed.quantize4(w, new(Ng, Nk, 16 * Nb), new(Ng, Nk, Nb))

    def run():
        xc, xs = routed.quantize4(x, new(Np, 16 * Nb), new(Np, Nb))
        o = OUT["bf16"]
        return (routed.group_fwd4(x, k, s, _out(Np, Nk, o), off),
                routed.group_fwd4(xc, k, s, _out(Np, Nk, o), off, InScales=xs),
                routed.group_bwd_in4(d, k, s, _out(Np, Nc, o), off))

    clean = run()
    for t in clean:
        assert torch.isfinite(t).all() and (t[P:] == 0).all()
    lo, hi = int(off[3]), int(off[4])
    s[3, 5, 2] = 255
    x[1], d[2] = math.nan, math.inf
    x[P:], d[P:] = math.nan, math.nan
    for i, t in enumerate(run()):
        bad = torch.zeros_like(t, dtype=torch.bool)
        if i < 2:
            bad[1], bad[lo:hi, 5] = True, True
        else:
            bad[2], bad[lo:hi, 64:96] = True, True
        assert torch.equal(t[~bad], clean[i][~bad])
        assert torch.isnan(t[lo:hi, 5] if i < 2 else t[lo:hi, 64:96]).all()
        assert not torch.isfinite(t[1 if i < 2 else 2]).any()


@pytest.mark.parametrize("Np", [2, 70, 700])
def test_ker_past_32_bits(Np):
    """The last group's Ker begins 4.9 GB into the tensor."""
    say(f"[group4 past 32 bits] {Np}")
    Ng, Nk, Nc = 300, 16392, 2048
    gen = torch.Generator().manual_seed(Np)
    codes, scales = four_bits.random(gen, 1, Nk, Nc=Nc)
    Ker = torch.empty((Ng, Nk, Nc // 2), dtype=torch.uint8, device="cuda")
    KerScales = torch.empty((Ng, Nk, Nc // 32), dtype=torch.uint8, device="cuda")
    Ker[-1], KerScales[-1] = codes[0].cuda(), scales[0].cuda()
    offsets = torch.zeros(Ng + 1, dtype=torch.int32)
    offsets[-1] = Np
    ker = four_bits.values(codes, scales, Nc)[0]
    x, d = _whole(gen, Np, Nc), _whole(gen, Np, Nk, top=1)
    got = routed.group_fwd4(x.cuda(), Ker, KerScales, _out(Np, Nk, torch.float32), offsets.cuda())
    assert torch.equal(got.cpu().double(), x.double() @ ker.t())
    xc, xs = four_bits.random(gen, Np, Nc=Nc)
    got = routed.group_fwd4(xc.cuda(), Ker, KerScales, _out(Np, Nk, torch.float32), offsets.cuda(), InScales=xs.cuda())
    assert torch.equal(got.cpu().double(), four_bits.values(xc, xs, Nc) @ ker.t())
    d[:, 2000:] = 0  # sums stay whole numbers in fp32
    d[:, -300:] = 1
    got = routed.group_bwd_in4(d.cuda(), Ker, KerScales, _out(Np, Nc, torch.float32), offsets.cuda())
    assert torch.equal(got.cpu().double(), d.double() @ ker)


@pytest.mark.parametrize("both", [False, True])
@pytest.mark.parametrize("Np", [5, 600])
def test_rows_past_31_bits(both, Np):
    """Gathered rows of an In of more than 2^31 bytes."""
    say(f"[group4 rows past 31 bits] {both} {Np}")
    Nt, Nc, Nk = ((1 << 22) + 5, 1024, 264) if both else ((1 << 20) + 7, 1040, 264)
    gen = torch.Generator().manual_seed(Np)
    codes, scales = four_bits.random(gen, 2, Nk, Nc=Nc)
    rows = torch.randperm(Nt, generator=gen)[:Np]
    rows[0], rows[1], rows[2] = Nt - 1, 0, Nt - 2
    if both:
        xc, xs = four_bits.random(gen, Np, Nc=Nc)
        x = four_bits.values(xc, xs, Nc)
        In = torch.empty((Nt, Nc // 2), dtype=torch.uint8, device="cuda")
        InScales = torch.empty((Nt, Nc // 32), dtype=torch.uint8, device="cuda")
        In[rows.cuda()], InScales[rows.cuda()] = xc.cuda(), xs.cuda()
        assert In.numel() > 1 << 31
    else:
        x, InScales = _whole(gen, Np, Nc), None
        In = torch.empty((Nt, Nc), dtype=torch.bfloat16, device="cuda")
        In[rows.cuda()] = x.cuda()
        assert In.numel() * 2 > 1 << 31
    offsets = torch.tensor([0, Np // 2, Np], dtype=torch.int32)
    got = routed.group_fwd4(In, codes.cuda(), scales.cuda(), _out(Np, Nk, torch.float32), offsets.cuda(),
                            rows.int().cuda(), InScales=InScales)
    assert torch.equal(got.cpu().double(), _product(x.double(), four_bits.values(codes, scales, Nc), offsets))


def test_one_ker_past_31_bits():
    """One group's Ker has more than 2^31 bytes of codes: zeros but for its ends."""
    say("[group4 one Ker past 31 bits]")
    Np, Nk, Nc, n = 5, (1 << 21) + 24, 2048, 50
    gen = torch.Generator().manual_seed(1)
    ends = [four_bits.random(gen, 1, n, Nc=Nc) for _ in range(2)]
    Ker = torch.zeros((1, Nk, Nc // 2), dtype=torch.uint8, device="cuda")
    KerScales = torch.full((1, Nk, Nc // 32), 127, dtype=torch.uint8, device="cuda")
    for (c, s), at in zip(ends, (slice(0, n), slice(Nk - n, Nk))):
        Ker[:, at], KerScales[:, at] = c.cuda(), s.cuda()
    ker = torch.cat([four_bits.values(c, s, Nc)[0] for c, s in ends])
    offsets = torch.tensor([0, Np], dtype=torch.int32)
    x, d = _whole(gen, Np, Nc), _whole(gen, Np, Nk)
    got = routed.group_fwd4(x.cuda(), Ker, KerScales, _out(Np, Nk, torch.float32), offsets.cuda())
    want = x.double() @ ker.t()
    assert torch.equal(got[:, :n].cpu().double(), want[:, :n]) and torch.equal(got[:, -n:].cpu().double(), want[:, n:])
    assert not got[:, n:-n].any()
    got = routed.group_bwd_in4(d.cuda(), Ker, KerScales, _out(Np, Nc, torch.float32), offsets.cuda())
    assert torch.equal(got.cpu().double(), torch.cat([d[:, :n], d[:, -n:]], 1).double() @ ker)


def test_rows_that_are_not_there():
    """Rows outside In read as zeros; offsets that are no order write nothing outside."""
    gen = torch.Generator().manual_seed(2)
    codes, scales = four_bits.random(gen, 2, 40, Nc=96)
    x = _whole(gen, 10, 96)
    xc, xs = four_bits.random(gen, 10, Nc=96)
    rows = torch.tensor([0, 9, 10, -3, 1 << 30, 4, -(1 << 31), 3], dtype=torch.int32)
    off = torch.tensor([0, 5, 8], dtype=torch.int32)
    there = ((rows >= 0) & (rows < 10))[:, None]
    for v, a, kw in ((x.double(), x, {}), (four_bits.values(xc, xs, 96), xc, {"InScales": xs.cuda()})):
        got = routed.group_fwd4(a.cuda(), codes.cuda(), scales.cuda(), _out(8, 40, torch.float32), off.cuda(),
                                rows.cuda(), **kw)
        want = _product(torch.where(there, v[rows.long().clamp(0, 9)], 0.0), four_bits.values(codes, scales, 96), off)
        assert torch.equal(got.double().cpu(), want)
        for bad in ([0, 9, 3], [0, -5, 8], [5, 5, 100000], [-(1 << 31), 0, (1 << 31) - 1]):
            o = torch.tensor(bad, dtype=torch.int32, device="cuda")
            out = _out(10, 40, torch.float32)
            routed.group_fwd4(a.cuda(), codes.cuda(), scales.cuda(), out[1:9], o, rows.cuda(), **kw)
            assert torch.isnan(out[0]).all() and torch.isnan(out[9]).all()


def test_stream_graph_and_repeat():
    """A graph of quantise, product of both in 4 bits, and gradient, replayed on new
    rows with other work between: every replay equals the plain calls bit for bit."""
    gen = torch.Generator().manual_seed(8)
    Nt, Nc, Nk, Ng = 300, 544, 200, 4
    codes, scales = (t.cuda() for t in four_bits.random(gen, Ng, Nk, Nc=Nc))
    off = torch.tensor([0, 100, 100, 230, 280], dtype=torch.int32, device="cuda")
    new = lambda *s: torch.empty(s, dtype=torch.uint8, device="cuda")  # noqa: E731
    x, xc, xs = torch.empty((Nt, Nc), dtype=torch.bfloat16, device="cuda"), new(Nt, 272), new(Nt, 17)
    outs = [_out(Nt, Nk, torch.bfloat16), _out(Nt, Nk, torch.float32), _out(Nt, Nc, torch.bfloat16), _out(Nt, Nc, torch.float32)]

    def step():
        routed.quantize4(x, xc, xs)
        routed.group_fwd4(xc, codes, scales, outs[0], off, InScales=xs)
        routed.group_fwd4(x, codes, scales, outs[1], off)
        routed.group_bwd_in4(outs[0], codes, scales, outs[2], off)
        routed.dequantize4(xc, xs, outs[3])

    data = [torch.randn((Nt, Nc), generator=gen).bfloat16() for _ in range(3)]
    want = []
    for v in data:
        x.copy_(v)
        step()
        want.append([o.clone() for o in outs])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want[-1]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in (0, 1, 2, 1, 0):
        x.copy_(data[i])
        for o in outs:
            o.fill_(math.nan)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want[i]))


def test_refusals():
    """The binding's own checks (the library's are tested without a GPU)."""
    u8 = lambda *s: torch.zeros(s, dtype=torch.uint8, device="cuda")  # noqa: E731
    x, xc, xs = torch.zeros((8, 64), dtype=torch.bfloat16, device="cuda"), u8(8, 32), u8(8, 2)
    k, s = u8(2, 4, 32), u8(2, 4, 2)
    off, out = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros((8, 4), device="cuda")
    d = out.bfloat16()
    fwd, bwd = routed.group_fwd4, routed.group_bwd_in4
    bad = [lambda: fwd(x.float(), k, s, out, off), lambda: fwd(xc, k, s, out, off), lambda: fwd(x.cpu(), k, s, out, off),
           lambda: fwd(x, k, s, out.half(), off), lambda: fwd(x, k[:, :, :16].contiguous(), s, out, off),
           lambda: fwd(x, k, s[:1], out, off), lambda: fwd(x, k, s.int(), out, off), lambda: fwd(x, k, s, out[:7], off),
           lambda: fwd(x, k, s, out, off.long()), lambda: fwd(x, k, s, out, off[:2]), lambda: fwd(x, k, s, out, off, off),
           lambda: fwd(x, k, s, out, off, InScales=xs), lambda: fwd(xc, k, s, out, off, InScales=xs[:7]),
           lambda: fwd(xc, k, s, out, off, InScales=xs.cpu()), lambda: fwd(xc, k.cpu(), s, out, off, InScales=xs),
           lambda: bwd(out, k, s, x, off), lambda: bwd(d, k, s, x[:7], off), lambda: bwd(d[:, :3].contiguous(), k, s, x, off),
           lambda: bwd(d, k, s, x.half(), off), lambda: bwd(d, k, s, x, off.long())]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    fwd(x, k, s, out, off)
    with pytest.raises(cnn.CnnError) as e:  # codes on no 16-byte boundary
        fwd(x, u8(300)[8:264].view(2, 4, 32), s, out, off)
    assert e.value.status == -2
    with pytest.raises(cnn.CnnError) as e:
        fwd(x, k, s, x.view(-1)[:32].view(8, 4), off)
    assert e.value.status == -5
