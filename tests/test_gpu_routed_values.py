"""Values that the routed contractions must keep: a low-rank factor of more bits
than two bf16 values hold, infinities that meet its parts, and gradients that are
not finite.

Whole numbers throughout, small enough that every sum is exact in fp32 in any
order: finite results are compared bit for bit."""
import math

import pytest
import torch

from gpu_helpers import say
from paper_2105_13480_amd import routed

pytestmark = pytest.mark.gpu

TYPES = {"f32": (torch.float32, torch.float32), "bf16": (torch.bfloat16, torch.float32),
         "bf16_obf16": (torch.bfloat16, torch.bfloat16)}
INF = math.inf

# rows, features in and out, adapters, ranks: rows as they come (100 rows), and in the
# order of their adapters by small tiles (whole units of ranks, and not; rows on no
# 4-byte boundary) and, in bf16, by 256 x 256 tiles
ADAPTED = [(100, 264, 328, 3, 8), (700, 264, 328, 3, 8), (700, 264, 328, 3, 7), (600, 515, 131, 3, 7),
           (5000, 1032, 2048, 3, 16)]


def _whole(gen, lo, hi, *shape):
    return torch.randint(lo, hi + 1, shape, generator=gen).float()


def _adapt(In, Ker, A, B, ids, to, scales=None):
    out = torch.full((In.shape[0], Ker.shape[0]), math.nan, dtype=to, device="cuda")
    i, k, a, b = In.cuda(), Ker.cuda(), A.cuda(), B.cuda()
    ws = routed.adapt_workspace(i, k, a, out)
    ws.fill_(0xff)  # NaN in every type
    routed.adapt_fwd(i, k, a, b, ids.cuda(), out, None if scales is None else scales.cuda(), ws)
    return out.cpu()


@pytest.mark.parametrize("mode", TYPES)
@pytest.mark.parametrize("case", ADAPTED, ids=str)
def test_low_rank_factor_in_full(case, mode):
    """The inner sum has up to 23 bits and the projection takes all but a few of
    them away again: what is left shows every bit that was not kept."""
    say(f"[factor] {case} {mode}")
    Nt, Nc, Nk, Na, Nl = case
    ti, to = TYPES[mode]
    gen = torch.Generator().manual_seed(Nt + Nl)
    In, A = _whole(gen, 0, 255, Nt, Nc), _whole(gen, 0, 31, 1, Nl, Nc)
    assert 255 * 32 * Nc < 1 << 24
    r, c = torch.arange(Nk) % Nl, torch.randint(0, Nc, (Nk,), generator=gen)
    Ker = -A[0][r]
    Ker[torch.arange(Nk), c] += 1  # Out: one value of In
    B = torch.zeros(Na, Nk, Nl)
    B[:, torch.arange(Nk), r] = 1
    ids = torch.randint(-1, Na, (Nt,), generator=gen).int()
    assert float((In @ A[0].t()).max()) > 1 << 18  # more than 17 bits
    want = torch.where((ids >= 0)[:, None], In[:, c], In @ Ker.t())
    got = _adapt(In.to(ti), Ker.to(ti), A.expand(Na, Nl, Nc).contiguous().to(ti), B.to(ti), ids, to)
    assert torch.equal(got, want.to(to))


def _products(x, y):
    """x y^T in 64 bits, infinities and NaN as each product gives them."""
    return torch.cat([(t[:, None] * y[None]).sum(2) for t in x.split(32)]) if len(x) else x @ y.t()


def _same(got, want):
    """Bit for bit, NaN where NaN is due."""
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(got, nan=0.0, posinf=INF, neginf=-INF),
                       torch.nan_to_num(want, nan=0.0, posinf=INF, neginf=-INF))


@pytest.mark.parametrize("mode", TYPES)
@pytest.mark.parametrize("case", ADAPTED, ids=str)
def test_adapters_of_infinite_weights(case, mode):
    """An infinite B times a finite factor other than zero is infinite, times
    zero NaN; an infinite factor is as the definition has it.  However many rows
    the call has."""
    say(f"[infinite] {case} {mode}")
    Nt, Nc, Nk, Na, Nl = case
    ti, to = TYPES[mode]
    gen = torch.Generator().manual_seed(Nt * 3 + Nl)
    In, Ker = _whole(gen, -2, 2, Nt, Nc), _whole(gen, -2, 2, Nk, Nc)
    A, B = _whole(gen, -1, 1, Na, Nl, Nc), _whole(gen, -1, 1, Na, Nk, Nl)
    B[0, 5, 2], B[0, 6, 0], B[0, 7, 1] = INF, -INF, math.nan
    B[0, Nk - 1, 3], B[0, Nk - 1, 4] = INF, -INF
    A[1, 3, 0] = INF      # the factor is infinite, or NaN where In[:, 0] is zero
    B[1, 9, 3] = INF
    B[1, 10] = 0
    ids = torch.randint(-1, Na, (Nt,), generator=gen).int()
    want = In.double() @ Ker.double().t()
    for a in range(Na):
        t = torch.nonzero(ids == a).reshape(-1)
        want[t] += _products(_products(In[t].double(), A[a].double()), B[a].double())
    got = _adapt(In.to(ti), Ker.to(ti), A.to(ti), B.to(ti), ids, to)
    _same(got.double(), want.float().to(to).double())


@pytest.mark.parametrize("mode", TYPES)
@pytest.mark.parametrize("over", ["all", "chosen"])
@pytest.mark.parametrize("Nt,Ng,Kt", [(5, 6, 2), (40, 200, 4), (17, 700, 8)])
def test_route_bwd_of_infinite_gradients(Nt, Ng, Kt, over, mode):
    """A weight's gradient that is not finite reaches neither the experts that are
    not allowed nor, over the chosen ones, those not chosen: theirs is zero."""
    say(f"[route_bwd infinite] {Nt} {Ng} {Kt} {over} {mode}")
    ti, to = TYPES[mode]
    gen = torch.Generator().manual_seed(Ng)
    logits = torch.randn((Nt, Ng), generator=gen).to(ti)
    logits[torch.rand((Nt, Ng), generator=gen) < 0.2] = -INF
    logits[1, : Ng // 2] = math.nan
    logits[:3, -2:] = 0.5  # two allowed at least
    barred = ~(logits.float() > -INF)
    r = routed.route(logits.cuda(), routed.Routing(Nt, Ng, Kt), over=over)
    choice = r.choice.cpu().long()
    dG = torch.randn((Nt, Kt), generator=gen)
    clean, dirty = (torch.full((Nt, Ng), math.nan, dtype=to, device="cuda") for _ in range(2))
    routed.route_bwd(logits.cuda(), r.choice, r.gates, dG.cuda(), clean, over=over)
    dG[0, 0], dG[1, 1], dG[2] = INF, math.nan, -INF
    routed.route_bwd(logits.cuda(), r.choice, r.gates, dG.cuda(), dirty, over=over)
    clean, dirty = clean.float().cpu(), dirty.float().cpu()
    outside = barred
    if over == "chosen":
        outside = torch.ones((Nt, Ng), dtype=torch.bool)
        outside.scatter_(1, choice.clamp(min=0), False)  # every row has a choice
    for d in (clean, dirty):
        assert (d[outside] == 0).all()
        assert not torch.signbit(d[outside]).any()  # not -0 either
    assert torch.equal(clean[3:], dirty[3:])
    assert not torch.isfinite(dirty[:3]).all(1).any()
