"""The router's balance on the GPU, against its definition in 64 bits on the CPU
with gradients by automatic differentiation.

Tolerances count roundings of 2^-24: p of a row of Ng experts is off by (Ng + 24 + the
largest |l - max| that still has weight) of them relative to itself (the difference's
rounding times the exponential's slope, the exponential and the division to some
units, the sum of Ng terms); a sum of T terms by T more; log-sum-exp by (Ng + 8) of
1 + |max| + log Ng."""
import math

import pytest
import torch

from gpu_helpers import say
from paper_2105_13480_amd import cnn, routed

pytestmark = pytest.mark.gpu

TYPES = {"f32": (torch.float32, torch.float32), "bf16": (torch.bfloat16, torch.float32),
         "bf16_obf16": (torch.bfloat16, torch.bfloat16)}
INF = math.inf
EPS = 2.0 ** -24


def _choice(logits, Kt):
    value, index = torch.sort(torch.nan_to_num(logits.double(), -INF, INF, -INF), dim=1, descending=True, stable=True)
    return torch.where(value[:, :Kt] > -INF, index[:, :Kt], -1).int()


def _oracle(logits, choice, bounds, d):
    """Counts, tokens, losses, gradient, and the magnitudes that the tolerances go by."""
    Nt, Ng = logits.shape
    Ns = len(bounds) - 1
    x = logits.double()
    x = torch.where(x > -INF, x, torch.full_like(x, -INF))  # NaN as -inf
    x.requires_grad_()
    counts, tokens = torch.zeros((Ns, Ng), dtype=torch.int32), torch.zeros(Ns, dtype=torch.int32)
    parts, squares, sizes = [], [], []
    weight = torch.zeros(Nt, dtype=torch.float64)
    shares = torch.zeros((Nt, Ng), dtype=torch.float64)
    z = torch.zeros(Nt, dtype=torch.float64)
    for s in range(Ns):
        live = []
        for t in range(bounds[s], bounds[s + 1]):
            some = False
            for e in choice[t].tolist():
                if 0 <= e < Ng:
                    counts[s, e] += 1
                    some = True
            if some and bool((x[t] > -INF).any()):
                live.append(t)
        tokens[s] = len(live)
        if not live:
            continue
        f = counts[s].double() / counts[s].sum()
        finite = x[live].amax(1) < INF
        p = torch.stack([torch.softmax(x[t], 0) if x[t].max() < INF else
                         (x[t].detach() == INF).double() / (x[t] == INF).sum() for t in live])
        lse = torch.logsumexp(x[live], 1)
        parts.append(Ng * (f * p.mean(0)).sum())
        squares += [l * l for l in lse]
        z[live] = lse.detach()
        weight[live] = Ng / len(live)
        shares[live] = f
        sizes += [float(v) for v in x[live].detach().amax(1)]
        assert finite.all() or not d.any()
    loss = torch.zeros(2, dtype=torch.float64)
    if parts:
        both = torch.stack([torch.stack(parts).mean(), torch.stack(squares).mean()])
        loss = both.detach()
        if d.any():
            (both * d.double()).sum().backward()
    grad = torch.zeros_like(x) if x.grad is None else torch.nan_to_num(x.grad)
    with torch.no_grad():
        p = torch.nan_to_num(torch.softmax(x, 1)) * (weight > 0)[:, None]
        mag = (d[0].double() * weight / max(1, len(parts)))[:, None] * p * (shares + (p * shares).sum(1, keepdim=True))
        m = torch.nan_to_num(x.amax(1), 0.0, 0.0, 0.0).abs()
        mag = mag + (2 * d[1].double() / max(1, int(tokens.sum())) * (1 + m + math.log(Ng)))[:, None] * p
    return counts, tokens, loss, grad.detach(), mag, z, m


def _check(logits, choice, bounds, mode, add=False, d=(0.7, 0.3), fill=0xff):
    Nt, Ng = logits.shape
    _, to = TYPES[mode]
    Kt = choice.shape[1]
    edges = [0, Nt] if bounds is None else bounds
    Ns = len(edges) - 1
    d = torch.tensor(d)
    counts, tokens, loss, grad, mag, z, m = _oracle(logits, choice, edges, d)
    x, c = logits.cuda(), choice.cuda()
    b = None if bounds is None else torch.tensor(bounds, dtype=torch.int32, device="cuda")
    n = torch.full((Ns, Ng), -7, dtype=torch.int32, device="cuda")
    t = torch.full((Ns,), -7, dtype=torch.int32, device="cuda")
    l = torch.full((2,), math.nan, device="cuda")
    ws = routed.balance_workspace(Nt, Ng, Ns)
    if ws is not None:
        ws.fill_(fill)
    routed.balance(x, c, n, t, l, b, ws)
    assert torch.equal(n.cpu(), counts) and torch.equal(t.cpu(), tokens)
    got = l.double().cpu()
    span = 110.0  # exp(-104) is the least weight of fp32
    T = int(tokens.sum())
    assert abs(got[0] - loss[0]) <= (2 * Ng + T + Ns + 32 + span) * EPS * loss[0]
    zerr = (Ng + 8) * EPS * (1 + m + math.log(Ng))
    tol = float(((2 * z.abs() + zerr) * zerr).sum()) / max(1, T) + (T + Ns + 8) * EPS * loss[1]
    assert abs(got[1] - loss[1]) <= tol
    old = torch.randn((Nt, Ng), generator=torch.Generator().manual_seed(1)).to(to)
    out = old.cuda() if add else torch.full((Nt, Ng), math.nan, dtype=to, device="cuda")
    routed.balance_bwd(x, c, n, t, d.cuda(), out, b, add=add)
    want = grad + old.double() if add else grad
    tol = (3 * Ng + 64 + span) * EPS * mag + EPS * want.abs()
    if to is torch.bfloat16:
        tol = tol + 2.0 ** -8 * (want.abs() + tol)
    bad = ~((out.double().cpu() - want).abs() <= tol + 1e-40)
    assert not bad.any(), (torch.nonzero(bad)[0], out.cpu()[bad][0], want[bad][0], tol[bad][0])


SHAPES = [(1, 1, 1), (1, 4, 4), (3, 7, 2), (65, 33, 5), (256, 32, 4), (257, 64, 8), (517, 130, 8), (130, 256, 16),
          (67, 257, 3), (300, 1024, 16), (1100, 16, 2)]


@pytest.mark.parametrize("mode", TYPES)
@pytest.mark.parametrize("Nt,Ng,Kt", SHAPES)
def test_one_sequence(Nt, Ng, Kt, mode):
    say(f"[balance] {Nt} {Ng} {Kt} {mode}")
    gen = torch.Generator().manual_seed(Nt + Ng)
    logits = (torch.randn((Nt, Ng), generator=gen) * 3).to(TYPES[mode][0])
    choice = _choice(logits, Kt)
    if Nt > 2:
        choice[Nt // 2] = -1            # a row that no expert takes
        choice[1, -1] = Ng + 3          # no expert
        choice[0] = choice[0, 0].clone()  # the same one again and again
    _check(logits, choice, None, mode, add=Nt % 2 == 0)


@pytest.mark.parametrize("mode", TYPES)
@pytest.mark.parametrize("Nt,Ng,Kt,bounds", [
    (40, 8, 2, [0, 40]), (40, 8, 2, [3, 3, 17, 17, 17, 30, 30]), (200, 24, 3, [0, 1, 2, 3, 64, 65, 128, 200]),
    (300, 65, 4, [0, 0, 300, 300]), (300, 12, 1, [299, 300]), (64, 16, 2, [64, 64, 64]), (1000, 40, 4, [7, 130, 131, 640, 990]),
    (150, 300, 2, [0, 70, 140])], ids=str)
def test_sequences(Nt, Ng, Kt, bounds, mode):
    """Empty ones, ones of a row, borders inside a workgroup's rows and on them,
    rows before the first and past the last."""
    say(f"[balance] {Nt} {Ng} {Kt} {bounds} {mode}")
    gen = torch.Generator().manual_seed(Nt + Ng)
    logits = torch.randn((Nt, Ng), generator=gen).to(TYPES[mode][0])
    logits[torch.rand((Nt, Ng), generator=gen) < 0.2] = -INF
    choice = _choice(logits, Kt)
    for add in (False, True):
        _check(logits, choice, bounds, mode, add)


def test_many_sequences():
    say("[balance] many")
    gen = torch.Generator().manual_seed(2)
    Nt, Ng = 3000, 20
    bounds = [0] + torch.sort(torch.randint(0, Nt, (700,), generator=gen)).values.tolist() + [2990]
    bounds = sorted(min(b, 2990) for b in bounds)
    logits = torch.randn((Nt, Ng), generator=gen)
    _check(logits, _choice(logits, 3), bounds, "f32")


@pytest.mark.parametrize("mode", TYPES)
def test_masks(mode):
    """Rows barred from some or all experts, lowest values, NaN, rows of one expert;
    all rows out: losses and gradient are zero."""
    say(f"[balance] masks {mode}")
    ti = TYPES[mode][0]
    low = torch.finfo(ti).min
    rows = [[-INF] * 6, [-INF, 1.0, -INF, -INF, -INF, -INF], [low, -INF, low, 0.0, low, -INF], [math.nan] * 6,
            [math.nan, 2.0, math.nan, -3.0, 2.0, 1.0], [-0.0, 0.0, -0.0, 0.0, -1.0, 1.0], [80.0, -80.0, 3.0, -3.0, 0.0, 1.0],
            [-80.0, 20.0, -200.0, 20.0, 19.0, -1e4]]
    logits = torch.tensor(rows * 9).to(ti)
    _check(logits, _choice(logits, 3), None, mode)
    _check(logits, _choice(logits, 3), [0, 8, 30, 72], mode, add=True)
    _check(logits, torch.full((72, 3), -1, dtype=torch.int32), [0, 8, 30, 72], mode)
    gone = torch.full((72, 6), -INF).to(ti)
    _check(gone, torch.zeros((72, 2), dtype=torch.int32), [0, 8, 30, 72], mode)


def test_infinite_logits_stay_in_their_row():
    """+inf takes the whole weight, shared with its kind; the loss on the size is then
    infinite, the balance is not, and other rows keep their gradient."""
    gen = torch.Generator().manual_seed(5)
    x = torch.randn((70, 9), generator=gen)
    x[4, 2] = x[4, 5] = x[9, 0] = INF
    choice = _choice(x, 2)
    n, t, l = torch.empty((1, 9), dtype=torch.int32, device="cuda"), torch.empty(1, dtype=torch.int32, device="cuda"), \
        torch.empty(2, device="cuda")
    routed.balance(x.cuda(), choice.cuda(), n, t, l)
    _, _, loss, *_ = _oracle(x, choice, [0, 70], torch.zeros(2))
    assert abs(float(l[0]) - float(loss[0])) <= 300 * EPS * float(loss[0]) and float(l[1]) == INF
    out = torch.empty((70, 9), device="cuda")
    routed.balance_bwd(x.cuda(), choice.cuda(), n, t, torch.tensor([1.0, 0.5], device="cuda"), out)
    g = out.cpu()
    others = [i for i in range(70) if i not in (4, 9)]
    assert torch.isfinite(g[others]).all() and (g[others] != 0).any(1).all()
    assert (g[4][[0, 1, 3, 4, 6, 7, 8]] == 0).all() and (g[9][1:] == 0).all()


def test_gradient_differences():
    """Against differences of the losses themselves."""
    gen = torch.Generator().manual_seed(3)
    x = torch.randn((6, 5), generator=gen)
    choice, b = _choice(x, 2).cuda(), torch.tensor([0, 4, 6], dtype=torch.int32, device="cuda")
    n, t = torch.empty((2, 5), dtype=torch.int32, device="cuda"), torch.empty(2, dtype=torch.int32, device="cuda")
    d = torch.tensor([0.6, 0.4], device="cuda")

    def losses(v):
        return routed.balance(v.cuda(), choice, n, t, torch.empty(2, device="cuda"), b).double().cpu()

    losses(x)
    g = routed.balance_bwd(x.cuda(), choice, n, t, d, torch.empty((6, 5), device="cuda"), b).cpu()
    h = 2.0 ** -7
    for i in range(6):
        for e in range(5):
            moved = torch.zeros_like(x)
            moved[i, e] = h
            up, down = losses(x + moved), losses(x - moved)
            diff = float(((up - down) * d.double().cpu()).sum()) / (2 * h)
            # third derivatives below 5 of each loss (h^2 / 6 of them), fp32 losses of size
            # below 16: 2^-24 16 (5 + 40) roundings / h
            assert abs(diff - float(g[i, e])) < 5 * h * h + 720 * EPS / h


def test_stream_graph_and_repeat():
    gen = torch.Generator().manual_seed(8)
    Nt, Ng, Kt, bounds = 900, 48, 4, [0, 300, 301, 880]
    b = torch.tensor(bounds, dtype=torch.int32, device="cuda")
    x = torch.empty((Nt, Ng), dtype=torch.bfloat16, device="cuda")
    c = torch.empty((Nt, Kt), dtype=torch.int32, device="cuda")
    n, t = torch.empty((3, Ng), dtype=torch.int32, device="cuda"), torch.empty(3, dtype=torch.int32, device="cuda")
    l, g, d = torch.empty(2, device="cuda"), torch.empty((Nt, Ng), device="cuda"), torch.tensor([0.1, 0.2], device="cuda")
    ws = routed.balance_workspace(Nt, Ng, 3)

    def step():
        routed.balance(x, c, n, t, l, b, ws)
        routed.balance_bwd(x, c, n, t, d, g, b)

    data, want = [], []
    for _ in range(3):
        v = torch.randn((Nt, Ng), generator=gen).bfloat16()
        data.append((v, _choice(v, Kt)))
        x.copy_(data[-1][0]), c.copy_(data[-1][1])
        step()
        want.append([o.clone() for o in (n, t, l, g)])
        # without a workspace, here and on a stream: the same
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        for stream in (None, side, side.cuda_stream):
            again = torch.full((2,), math.nan, device="cuda")
            torch.cuda.synchronize()
            routed.balance(x, c, n, t, again, b, stream=stream)
            torch.empty(1 << 20, dtype=torch.uint8, device="cuda").fill_(0xff)
            torch.cuda.synchronize()
            assert torch.equal(again, want[-1][2])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in (0, 1, 2, 1, 0):
        x.copy_(data[i][0]), c.copy_(data[i][1])
        for o in (n, t, l, g):
            o.fill_(-1)
        ws.fill_(0xee)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip((n, t, l, g), want[i]))


def test_bad_bounds_stay_inside():
    """Bounds that are no order give some result and write nothing else."""
    x = torch.randn((200, 8), device="cuda")
    c = torch.zeros((200, 2), dtype=torch.int32, device="cuda")
    for bad in ([5, 3, 1], [-100, 900, 200], [1 << 30, -5, 1 << 30], [0, 200, 0], [200, 0, 100]):
        n, t = torch.full((4, 8), -7, dtype=torch.int32, device="cuda"), torch.full((4,), -7, dtype=torch.int32, device="cuda")
        l, g = torch.full((4,), -7.0, device="cuda"), torch.full((202, 8), -7.0, device="cuda")
        b = torch.tensor(bad, dtype=torch.int32, device="cuda")
        routed.balance(x, c, n[1:3], t[1:3], l[1:3], b)
        routed.balance_bwd(x, c, n[1:3], t[1:3], l[1:3], g[1:201], b)
        assert (n[0] == -7).all() and (n[3] == -7).all() and t[0] == -7 == t[3] and l[0] == -7 == l[3]
        assert (g[0] == -7).all() and (g[201] == -7).all()


def test_no_rows_and_refusals():
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    x, c, n, t, l = torch.zeros((8, 6), device="cuda"), i32(8, 2), i32(1, 6), i32(1), torch.ones(2, device="cuda")
    n.fill_(5)
    routed.balance(x[:0], c[:0], n, t, l)
    assert (n == 0).all() and (t == 0).all() and (l == 0).all()
    routed.balance_bwd(x[:0], c[:0], n, t, l, x[:0].clone())
    f, b = routed.balance, routed.balance_bwd
    bad = [lambda: f(x.cpu(), c, n, t, l), lambda: f(x.t(), c, n, t, l), lambda: f(x.half(), c, n, t, l),
           lambda: f(x, c[:7], n, t, l), lambda: f(x, c.long(), n, t, l), lambda: f(x, c, n[:, :5].contiguous(), t, l),
           lambda: f(x, c, n, i32(2), l), lambda: f(x, c, n, t, l[:1]), lambda: f(x, c, n, t, l.double()),
           lambda: f(x, c, n, t, l, i32(3)), lambda: f(x, c, n, t, l, i32(2).long()), lambda: f(x, c, n, t, l, i32(2), ws=l.cpu()),
           lambda: b(x, c, n, t, l, x.bfloat16()), lambda: b(x, c, n, t, l, x[:7].clone()), lambda: b(x, c, n, t, l.cpu(), x.clone())]
    for g in bad:
        with pytest.raises(ValueError):
            g()
    with pytest.raises(cnn.CnnError) as e:  # two sequences without bounds
        f(x, c, i32(2, 6), i32(2), l)
    assert e.value.status == -2
    with pytest.raises(cnn.CnnError) as e:  # a workspace too small
        f(x, c, i32(2, 6), i32(2), l, i32(3), ws=torch.empty(16, dtype=torch.uint8, device="cuda"))
    assert e.value.status == -2
    with pytest.raises(cnn.CnnError) as e:
        b(x, c, n, t, l, x)
    assert e.value.status == -5
