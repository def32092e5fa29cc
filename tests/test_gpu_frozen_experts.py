"""The 4-bit contractions and the router's balance together, as a layer of routed
experts uses them: results and gradients against the same layer in 64 bits, eager
and captured into a graph.

A bf16 result is off by 2^-8 of itself; what it is multiplied with carries that on.
The bounds below add up these parts with the magnitudes of the products (fp32 sums
add less than 2^-12 of those at these sizes)."""
import math
import os
import sys

import pytest
import torch

import four_bits
from gpu_helpers import say

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import frozen_experts  # noqa: E402

pytestmark = pytest.mark.gpu

HALF, SUM = 2.0 ** -8, 2.0 ** -12


def _layer(rows, features, hidden, experts, choices, bounds, four):
    layer = frozen_experts.FrozenExperts(features, hidden, experts, choices, rows, len(bounds) - 1, four, seed=rows)
    gen = torch.Generator().manual_seed(features)
    In = torch.randn((rows, features), generator=gen).bfloat16()
    logits = torch.randn((rows, experts), generator=gen)
    logits[rows // 2] = -math.inf  # a row that goes nowhere
    dOut = torch.randn((rows, features), generator=gen).bfloat16()
    return layer, In, logits, dOut, torch.tensor(bounds, dtype=torch.int32), torch.tensor([0.3, 0.05])


def _near(got, want, tol):
    bad = ~((got.double().cpu() - want).abs() <= tol)
    assert not bad.any(), (int(bad.sum()), torch.nonzero(bad)[0].tolist(), got.cpu()[bad][0], want[bad][0], tol[bad][0])


CASES = [(1, 64, 32, 4, 2, [0, 1]), (40, 96, 130, 5, 2, [0, 7, 33]), (300, 515, 264, 8, 3, [0, 100, 100, 300]),
         (700, 544, 1000, 6, 1, [0, 650])]


@pytest.mark.parametrize("four", [True, False])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_against_64_bits(case, four):
    say(f"[frozen experts] {case} {four}")
    rows, features, hidden, experts, choices, _ = case
    layer, In, logits, dOut, bounds, dl = _layer(*case, four)
    Out, losses, kept = layer.forward(In.cuda(), logits.cuda(), bounds.cuda())
    dIn, dLogits = layer.backward(dOut.cuda(), dl.cuda(), kept)
    o = layer.order
    choice, K1 = o.choice.cpu().long(), four_bits.values(layer.K1.cpu(), layer.K1s.cpu(), features)
    K2 = four_bits.values(layer.K2.cpu(), layer.K2s.cpu(), hidden)
    x = In.double()
    if four:
        codes, scales = four_bits.quantize(In, "floor")
        x = four_bits.values(four_bits.pack(codes), scales, features)
    l = logits.double().requires_grad_()
    live = (choice >= 0).any(1)
    p = torch.zeros((rows, experts), dtype=torch.float64)
    p[live] = torch.softmax(l[live], 1)
    want, mag = torch.zeros((rows, features), dtype=torch.float64), torch.zeros((rows, features), dtype=torch.float64)
    dx, dmag = torch.zeros_like(want), torch.zeros_like(want)
    score, serr = torch.zeros((), dtype=torch.float64), torch.zeros((rows, experts), dtype=torch.float64)
    d = dOut.double()
    for t in range(rows):
        for e in choice[t].tolist():
            if e < 0:
                continue
            g = p[t, e]
            gd = float(g.detach())
            h = K1[e] @ x[t]
            herr = HALF * h.abs() + SUM * (K1[e].abs() @ x[t].abs())
            s = torch.relu(h) ** 2
            s_err = (torch.relu(h) + herr) ** 2 - s + HALF * (torch.relu(h) + herr) ** 2
            z = K2[e] @ s
            zerr = K2[e].abs() @ s_err + SUM * (K2[e].abs() @ s) + HALF * z.abs()
            zerr = zerr * (1 + HALF)
            want[t] += gd * z
            mag[t] += gd * zerr
            score = score + g * (d[t] @ z)
            serr[t, e] = d[t].abs() @ zerr + SUM * (d[t].abs() @ z.abs())
            dz, dzerr = gd * d[t], HALF * gd * d[t].abs() * 1.01
            ds = K2[e].t() @ dz
            dserr = K2[e].abs().t() @ dzerr + SUM * (K2[e].abs().t() @ dz.abs()) + HALF * ds.abs() * 1.1
            # 2 relu(h) is off where h is, and each product once more
            slope = 2 * (torch.relu(h) + herr)
            dh = ds * 2 * torch.relu(h)
            dherr = (slope * (1 + HALF) - 2 * torch.relu(h)) * (ds.abs() + dserr) + 2 * torch.relu(h) * dserr
            dherr = dherr + torch.where(h.abs() <= herr, slope * (ds.abs() + dserr), torch.zeros_like(dherr))
            dherr = (dherr + HALF * (dh.abs() + dherr)) * 1.01
            dp = K1[e].t() @ dh
            dperr = K1[e].abs().t() @ dherr + SUM * (K1[e].abs().t() @ dh.abs())
            dperr = dperr + HALF * (dp.abs() + dperr)
            dx[t] += dp
            dmag[t] += dperr
    _near(Out, want, mag + HALF * (want.abs() + mag) + 1e-30)
    _near(dIn, dx, dmag + HALF * (dx.abs() + dmag) + 1e-30)
    # the losses, and the gradient of all three through the logits
    total, squares, used, n = torch.zeros((), dtype=torch.float64), torch.zeros((), dtype=torch.float64), 0, 0
    b = bounds.tolist()
    for s in range(len(b) - 1):
        rows_s = [t for t in range(b[s], b[s + 1]) if live[t]]
        if rows_s:
            f = torch.bincount(choice[rows_s].reshape(-1), minlength=experts).double()
            total = total + experts * (f / f.sum() * p[rows_s].mean(0)).sum()
            squares = squares + (torch.logsumexp(l[rows_s], 1) ** 2).sum()
            used, n = used + 1, n + len(rows_s)
    total, squares = total / max(used, 1), squares / max(n, 1)  # no row takes part: zero
    assert abs(float(losses[0]) - float(total)) <= 1e-4 * float(total)
    assert abs(float(losses[1]) - float(squares)) <= 1e-4 * float(squares)
    (score + float(dl[0]) * total + float(dl[1]) * squares + 0 * torch.nan_to_num(l).sum()).backward()
    grad = torch.nan_to_num(l.grad)
    ge = (p.detach() * serr)
    tol = ge + p.detach() * ge.sum(1, keepdim=True) + SUM * (grad.abs() + p.detach()) * (1 + serr.sum(1, keepdim=True))
    _near(dLogits, grad, tol + 1e-30)


def test_captured():
    """Forward and backward captured and replayed on new rows, with other work between:
    every replay equals the plain calls bit for bit."""
    say("[frozen experts] captured")
    case = (500, 320, 264, 6, 2, [0, 111, 480])
    layer, In, logits, dOut, bounds, dl = _layer(*case, True)
    x, l, d, b, w = In.cuda(), logits.cuda(), dOut.cuda(), bounds.cuda(), dl.cuda()

    def step():
        out, losses, kept = layer.forward(x, l, b)
        return (out, losses, layer.counts, *layer.backward(d, w, kept))

    gen = torch.Generator().manual_seed(4)
    data = [(torch.randn(x.shape, generator=gen).bfloat16(), torch.randn(l.shape, generator=gen)) for _ in range(3)]
    want = []
    for v, m in data:
        x.copy_(v), l.copy_(m)
        want.append([t.clone() for t in step()])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for i in (0, 1, 2, 1, 0):
        x.copy_(data[i][0]), l.copy_(data[i][1])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want[i]))


def test_example_runs(capsys):
    frozen_experts.main(["--rows", "300", "--features", "256", "--hidden", "512", "--experts", "8", "--steps", "2"])
    assert "4 bits" in capsys.readouterr().out
