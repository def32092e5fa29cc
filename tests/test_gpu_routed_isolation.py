"""NaN and infinities stay in their adapter's or group's rows on the paths of many
rows (rows in the order of their adapters; 256 x 256 tiles), memory that no one
wrote stays out of results, and calls repeat bit for bit."""
import math

import pytest
import torch

from gpu_helpers import say
from paper_2105_13480_amd import routed

pytestmark = pytest.mark.gpu

TYPES = {"f32": (torch.float32, torch.float32), "bf16": (torch.bfloat16, torch.float32),
         "bf16_obf16": (torch.bfloat16, torch.bfloat16)}
INF = math.inf

# rows, features in and out, adapters, ranks: small tiles with whole units of ranks and
# not, rows on no 4-byte boundary, and in bf16 256 x 256 tiles with one run of ranks and two
ORDERED = [(700, 264, 328, 3, 8), (700, 264, 328, 3, 7), (2500, 515, 777, 4, 12), (1500, 264, 328, 70, 16),
           (5000, 1032, 2048, 3, 16), (8192, 1032, 2048, 5, 64)]


def _data(case, ti):
    Nt, Nc, Nk, Na, Nl = case
    gen = torch.Generator(device="cuda").manual_seed(Nt + Nl)
    new = lambda *s: torch.randn(s, generator=gen, device="cuda").to(ti)  # noqa: E731
    ids = torch.randint(-1, Na, (Nt,), generator=gen, device="cuda").int()  # boundaries anywhere in a tile
    return new(Nt, Nc), new(Nk, Nc), new(Na, Nl, Nc), new(Na, Nk, Nl), ids


def _adapt(In, Ker, A, B, ids, to, fill):
    out = torch.full((In.shape[0], Ker.shape[0]), math.nan, dtype=to, device="cuda")
    ws = routed.adapt_workspace(In, Ker, A, out)
    ws.fill_(fill)
    return routed.adapt_fwd(In, Ker, A, B, ids, out, None, ws)


@pytest.mark.parametrize("mode", TYPES)
@pytest.mark.parametrize("case", ORDERED, ids=str)
def test_adapters_in_order(case, mode):
    say(f"[adapters in order] {case} {mode}")
    ti, to = TYPES[mode]
    In, Ker, A, B, ids = _data(case, ti)
    clean = _adapt(In, Ker, A, B, ids, to, 0)
    assert torch.isfinite(clean).all()
    # what the workspace held (0xff: NaN) is in no result, of rows without an adapter neither
    assert torch.equal(_adapt(In, Ker, A, B, ids, to, 0xff), clean)
    for dirt in (lambda: A[1, 2].fill_(INF), lambda: B[1].fill_(math.nan), lambda: B[1, 5].fill_(-INF)):
        keep = A.clone(), B.clone()
        dirt()
        out = _adapt(In, Ker, A, B, ids, to, 0xff)
        assert torch.equal(out[ids != 1], clean[ids != 1])
        assert not torch.isfinite(out[ids == 1][:, 5]).any()
        A, B = keep


@pytest.mark.parametrize("mode", TYPES)
@pytest.mark.parametrize("case", [(48, 1024, 512, 5, 16)] + ORDERED, ids=str)
def test_adapters_repeat(case, mode):
    """Pass after pass, with passes on other rows between that nothing waits for."""
    say(f"[adapters repeat] {case} {mode}")
    ti, to = TYPES[mode]
    In, Ker, A, B, ids = _data(case, ti)
    first = _adapt(In, Ker, A, B, ids, to, 0)
    ws = [routed.adapt_workspace(In, Ker, A, first) for _ in range(2)]
    other = torch.empty_like(first)
    back = In.flip(0), ids.flip(0)
    for _ in range(4):
        again = torch.full_like(first, math.nan)
        routed.adapt_fwd(back[0], Ker, A, B, back[1], other, None, ws[1])
        routed.adapt_fwd(In, Ker, A, B, ids, again, None, ws[0])
        routed.adapt_fwd(back[0], Ker, A, B, back[1], other, None, ws[1])
        assert torch.equal(again, first)


@pytest.mark.parametrize("gathered", [True, False])
@pytest.mark.parametrize("mode", TYPES)
def test_groups_in_large_tiles(mode, gathered):
    """Group 3 of NaN and infinities, and rows of none."""
    say(f"[groups in large tiles] {mode} {gathered}")
    ti, to = TYPES[mode]
    sizes, past, Nc, Nk = [1300, 57, 0, 901, 2400, 3], 43, 2048, 2056
    gen = torch.Generator(device="cuda").manual_seed(3)
    new = lambda *s: torch.randn(s, generator=gen, device="cuda").to(ti)  # noqa: E731
    off = torch.tensor([0] + sizes).cumsum(0).int().cuda()
    P, Np = sum(sizes), sum(sizes) + past
    In, Ker, dOut = new(Np, Nc), new(len(sizes), Nk, Nc), new(Np, Nk)
    rows = torch.randperm(Np, generator=gen, device="cuda").int() if gathered else None
    if gathered:
        rows[P:] = -1
    bad = slice(1357, 1357 + 901)  # group 3's places
    source = rows[bad].long() if gathered else torch.arange(Np, device="cuda")[bad]

    def run():
        e = lambda *s: torch.full(s, math.nan, dtype=to, device="cuda")  # noqa: E731
        return (routed.group_fwd(In, Ker, e(Np, Nk), off, rows), routed.group_bwd_in(dOut, Ker, e(Np, Nc), off),
                routed.group_bwd_ker(dOut, In, e(len(sizes), Nk, Nc), off, rows))

    clean = run()
    for t in clean:
        assert torch.isfinite(t).all()
    Ker[3, ::7] = math.nan
    In[source] = INF
    dOut[bad] = -INF
    dOut[P:] = math.nan
    if not gathered:
        In[P:] = math.nan
    keep = torch.ones(Np, dtype=torch.bool, device="cuda")
    keep[bad] = False
    fwd, bwd_in, bwd_ker = run()
    assert torch.equal(fwd[keep], clean[0][keep]) and not torch.isfinite(fwd[bad]).any()
    assert torch.equal(bwd_in[keep], clean[1][keep]) and not torch.isfinite(bwd_in[bad]).any()
    groups = torch.tensor([g != 3 for g in range(len(sizes))], device="cuda")
    assert torch.equal(bwd_ker[groups], clean[2][groups]) and not torch.isfinite(bwd_ker[3]).any()
