"""The routed contractions together (the example's layer against its definition
in 64 bits, its gradients against the definition's and against differences), and
each of them on every tile size with whole numbers, where every sum is exact:
results are compared bit for bit and gradients with differences of the forward
products themselves.

With whole numbers of magnitude at most 3 and at most 9000 products a sum, every
partial sum is a whole number below 2^24: exact in fp32 in any order."""
import importlib.util
import os

import pytest
import torch

from gpu_helpers import say
from paper_2105_13480_amd import routed

pytestmark = pytest.mark.gpu

TYPES = {"f32": (torch.float32, torch.float32), "bf16": (torch.bfloat16, torch.float32),
         "bf16_obf16": (torch.bfloat16, torch.bfloat16)}
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("routed_layer",
                                                  os.path.join(ROOT, "examples", "routed_layer.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


# ---- the layer ---------------------------------------------------------------

def _plain(p, scales, In, ids, choice, over):
    """The layer of one type's parameters in 64 bits, with the choice given."""
    y = In @ p["W"].t()
    low = torch.zeros_like(y)
    for a in range(p["A"].shape[0]):
        rows = torch.nonzero(ids == a)[:, 0]
        low = low.index_add(0, rows, scales[a] * (In[rows] @ p["A"][a].t()) @ p["B"][a].t())
    y = y + low
    logits = y @ p["R"][0].t()
    chosen = torch.gather(logits, 1, choice)
    gates = torch.softmax(chosen, 1) if over == "chosen" else torch.gather(torch.softmax(logits, 1), 1, choice)
    out = torch.zeros_like(y)
    for e in range(p["K1"].shape[0]):
        t, j = torch.nonzero(choice == e, as_tuple=True)
        z = torch.relu(y[t] @ p["K1"][e].t()).square() @ p["K2"][e].t()
        out = out.index_add(0, t, gates[t, j][:, None] * z)
    return out


# rows, features, hidden, experts, choices, adapters, ranks
LAYERS = [(1, 64, 32, 4, 2, 2, 8), (7, 33, 20, 3, 3, 1, 5), (50, 64, 64, 8, 2, 3, 16),
          (300, 96, 40, 5, 1, 4, 4)]


@pytest.mark.parametrize("over", ["all", "chosen"])
@pytest.mark.parametrize("case", LAYERS, ids=str)
def test_layer_and_gradients(case, over):
    """fp32.  A result passes through at most ten products of at most 100
    factors (50 for the sums over rows, which start from smaller values); each
    adds at most (100 + 8) 2^-24 of its absolute sum, which is at most
    sqrt(100) of the result's norm for values of random sign: 10 x 108 x 10 x
    2^-24 = 6.5e-4 of the norm."""
    say(f"[layer] {case} {over}")
    N, C, H, E, K, Na, Nl = case
    layer = _example().RoutedLayer(C, H, E, K, Na, Nl, N, dtype=torch.float32, over=over, seed=N)
    gen = torch.Generator().manual_seed(N + 1)
    In, dOut = torch.randn((N, C), generator=gen), torch.randn((N, C), generator=gen)
    ids = torch.randint(-1, Na + 1, (N,), generator=gen).int()  # both ends: no adapter
    out, kept = layer.forward(In.cuda(), ids.cuda())
    dIn, grad = layer.backward(dOut.cuda(), kept)

    p = {n: t.double().cpu().requires_grad_() for n, t in layer.parameters().items()}
    x = In.double().requires_grad_()
    scales, choice = layer.scales.double().cpu(), layer.order.choice.long().cpu()
    want = _plain(p, scales, x, ids, choice, over)
    (want * dOut.double()).sum().backward()

    def near(name, got, exact):
        off = float((got.double().cpu() - exact).norm())
        assert off <= 6.5e-4 * float(exact.norm()) + 1e-12, f"{name}: off by {off} of {float(exact.norm())}"

    near("Out", out, want.detach())
    near("dIn", dIn, x.grad)
    for n in p:
        exact = p[n].grad if p[n].grad is not None else torch.zeros_like(p[n])
        near(n, grad[n], exact)

    # differences of the definition, along the kernels' own gradient
    with torch.no_grad():
        for n, g in list(grad.items()) + [("In", dIn)]:
            g = g.double().cpu()
            size = float(g.norm())
            if size == 0:
                continue
            v, f = g / size, []
            for h in (1e-5, -1e-5):
                q = dict(p)
                moved = x
                if n == "In":
                    moved = x + h * v
                else:
                    q[n] = p[n] + h * v
                f.append(float((_plain(q, scales, moved, ids, choice, over) * dOut.double()).sum()))
            slope = (f[0] - f[1]) / 2e-5
            # the kernels' bound, and the definition's rounding over the step
            assert abs(slope - size) <= 1e-3 * size + 1e-15 * abs(f[0]) / 1e-5 * 100, (n, slope, size)


def test_layer_in_a_graph():
    """A captured step gives the eager step's results, replay after replay."""
    layer = _example().RoutedLayer(64, 128, 8, 2, 3, 8, 40)
    gen = torch.Generator().manual_seed(2)
    In, dOut = (torch.randn((40, 64), generator=gen).bfloat16().cuda() for _ in range(2))
    ids = torch.randint(-1, 3, (40,), generator=gen).int().cuda()
    out, kept = layer.forward(In, ids)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        layer.forward(In, ids)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        again, _ = layer.forward(In, ids)
    for seed in range(3):
        In.copy_(torch.randn((40, 64), generator=torch.Generator().manual_seed(seed)).bfloat16())
        eager, _ = layer.forward(In, ids)
        eager = eager.clone()
        again.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(again, eager)


def test_example_runs(capsys):
    _example().main(["--rows", "256", "--features", "128", "--hidden", "192", "--steps", "2"])
    assert "forward" in capsys.readouterr().out


# ---- whole numbers: every tile size, exactly ---------------------------------

# rows of the groups (the rest of the places have none), features in and out,
# rows past the last group: the large tiles with long and short last tiles, more
# groups than a wave has lanes, more rows of a group than are held at a time,
# then the smaller tiles, aligned and not
SIZES = [([9000, 4200], 2056, 2064, 0), ([5000, 0, 4201, 57, 1], 2056, 1544, 90),
         ([160] * 66 + [0, 700], 520, 1288, 3), ([700, 0, 600, 1, 256, 900], 520, 1024, 5),
         ([513, 300], 1032, 776, 0), ([40] * 70 + [300, 0, 1], 264, 200, 130),
         ([130, 0, 77, 250], 264, 640, 1), ([130, 0, 77, 250], 263, 129, 1),
         ([20, 9, 31, 0, 12], 136, 72, 2), ([20, 9, 31, 0, 12], 35, 71, 2),
         ([3] * 9 + [7], 1032, 104, 0), ([33], 2048, 1, 0), ([0, 1, 0], 1, 512, 0),
         # rows shorter than 16 bytes, ends inside 16 bytes, odd sizes in large tiles
         ([300, 0, 41], 5, 3, 4), ([300, 41], 7, 1023, 0), ([90] * 3, 1023, 5, 1), ([150, 80], 9, 11, 0),
         ([700, 0, 400], 2047, 130, 3), ([1500, 300], 515, 2049, 0)]


def _whole(gen, *shape, top=2, dtype=torch.float32):
    return torch.randint(-top, top + 1, shape, generator=gen).to(dtype)


def _name(case):
    g, Nc, Nk, past = case
    return f"{len(g)}x{sum(g)}-{Nc}-{Nk}-{past}"


def _product(case, mode):
    sizes, Nc, Nk, past = case
    ti, _ = TYPES[mode]
    gen = torch.Generator().manual_seed(len(sizes) * 1000 + Nc)
    P = sum(sizes)
    offsets = torch.tensor([0] + sizes).cumsum(0).int()
    rows = torch.randperm(P + past, generator=gen).int()
    rows[P:] = -1
    In = _whole(gen, P + past, Nc, dtype=ti)
    return (offsets, rows, In, _whole(gen, len(sizes), Nk, Nc, dtype=ti),
            _whole(gen, P + past, Nk, dtype=ti))


@pytest.mark.parametrize("mode", TYPES)
@pytest.mark.parametrize("case", SIZES, ids=_name)
def test_products_exact(case, mode):
    say(f"[exact] {_name(case)} {mode}")
    _, to = TYPES[mode]
    offsets, rows, In, Ker, dOut = _product(case, mode)
    off, P, Np = offsets.tolist(), int(offsets[-1]), rows.numel()
    Ng, Nk, Nc = Ker.shape
    x = In[rows.long().clamp(min=0)].float()
    want = {"fwd": torch.zeros(Np, Nk), "in": torch.zeros(Np, Nc), "ker": torch.zeros(Ng, Nk, Nc)}
    for g in range(Ng):
        at = slice(off[g], off[g + 1])
        want["fwd"][at] = x[at] @ Ker[g].float().t()
        want["in"][at] = dOut[at].float() @ Ker[g].float()
        want["ker"][g] = dOut[at].float().t() @ x[at]
    new = lambda *shape: torch.full(shape, float("nan"), dtype=to, device="cuda")  # noqa: E731
    o, r, i, k, d = (t.cuda() for t in (offsets, rows, In, Ker, dOut))
    xs = i[r.long().clamp(min=0)]
    got = {"fwd": [routed.group_fwd(i, k, new(Np, Nk), o, r), routed.group_fwd(xs, k, new(Np, Nk), o)],
           "in": [routed.group_bwd_in(d, k, new(Np, Nc), o)],
           "ker": [routed.group_bwd_ker(d, i, new(Ng, Nk, Nc), o, r),
                   routed.group_bwd_ker(d, xs, new(Ng, Nk, Nc), o)]}
    for name, results in got.items():
        for result in results:
            assert torch.equal(result.cpu(), want[name].to(to)), name


def _loss(out, d):
    return float((out.double().cpu() * d.double()).sum())


@pytest.mark.parametrize("mode", ["f32", "bf16"])
@pytest.mark.parametrize("case", SIZES[3:], ids=_name)
def test_product_gradients_differences(case, mode):
    """The products are linear in each operand: with whole numbers a difference
    over any step equals the gradient along it exactly."""
    say(f"[differences] {_name(case)} {mode}")
    ti, _ = TYPES[mode]
    offsets, rows, In, Ker, dOut = _product(case, mode)
    gen = torch.Generator().manual_seed(5)
    vi, vk = _whole(gen, *In.shape, top=1, dtype=ti), _whole(gen, *Ker.shape, top=1, dtype=ti)
    Ng, Nk, Nc = Ker.shape
    Np = rows.numel()
    o, r = offsets.cuda(), rows.cuda()
    new = lambda *shape: torch.full(shape, float("nan"), device="cuda")  # noqa: E731
    fwd = lambda i, k: routed.group_fwd(i.cuda(), k.cuda(), new(Np, Nk), o, r)  # noqa: E731
    dk = routed.group_bwd_ker(dOut.cuda(), In.cuda(), new(Ng, Nk, Nc), o, r)
    assert _loss(fwd(In, Ker + vk), dOut) - _loss(fwd(In, Ker - vk), dOut) == 2 * _loss(dk, vk)
    # of a row: the sum over its places
    slots = torch.full((Np, 1), -1, dtype=torch.int32)
    P = int(offsets[-1])
    slots[rows[:P].long(), 0] = torch.arange(P).int()
    di = routed.group_bwd_in(dOut.cuda(), Ker.cuda(), new(Np, Nc), o)
    dx = routed.combine(di, new(Np, Nc), slots.cuda())
    assert _loss(fwd(In + vi, Ker), dOut) - _loss(fwd(In - vi, Ker), dOut) == 2 * _loss(dx, vi)


@pytest.mark.parametrize("mode", ["f32", "bf16"])
@pytest.mark.parametrize("Nt,Ng,Kt,Nk", [(1, 1, 1, 1), (7, 5, 3, 65), (33, 16, 4, 256), (300, 8, 2, 520)])
def test_combine_gradients_differences(Nt, Ng, Kt, Nk, mode):
    """Linear in its rows and in its weights (here eighths): exact as above."""
    say(f"[combine differences] {Nt} {Ng} {Kt} {Nk} {mode}")
    ti, _ = TYPES[mode]
    gen = torch.Generator().manual_seed(Nt)
    r = routed.route(torch.randn((Nt, Ng), generator=gen).cuda(), routed.Routing(Nt, Ng, Kt))
    In, vi = _whole(gen, Nt * Kt, Nk, dtype=ti), _whole(gen, Nt * Kt, Nk, top=1, dtype=ti)
    gates, vg = (torch.randint(-8, 9, (Nt, Kt), generator=gen) / 8.0 for _ in range(2))
    dOut = _whole(gen, Nt, Nk, dtype=ti)
    new = lambda *shape: torch.full(shape, float("nan"), device="cuda")  # noqa: E731
    f = lambda i, g: _loss(routed.combine(i.cuda(), new(Nt, Nk), r.slots, g.cuda()), dOut)  # noqa: E731
    dIn, dG = routed.combine_bwd(dOut.cuda(), In.cuda(), new(Nt * Kt, Nk), new(Nt, Kt), r.slots, r.rows,
                                 gates.cuda())
    assert f(In + vi, gates) - f(In - vi, gates) == 2 * _loss(dIn, vi)
    assert f(In, gates + vg) - f(In, gates - vg) == 2 * _loss(dG, vg)


@pytest.mark.parametrize("mode", ["f32", "bf16", "bf16_obf16"])
@pytest.mark.parametrize("Nt,Nc,Nk,Na,Nl", [(1, 1032, 520, 3, 8), (40, 264, 72, 70, 16), (300, 2056, 328, 5, 12),
                                            (700, 520, 640, 3, 40), (600, 515, 131, 4, 7), (1500, 264, 328, 2, 16),
                                            (4000, 264, 2080, 6, 8), (5000, 1032, 2048, 3, 16),
                                            (333, 1001, 153, 5, 12), (150, 1001, 77, 4, 9),
                                            (450, 2048, 2048, 3, 8), (9, 5, 3, 2, 2), (700, 1003, 259, 3, 64)])
def test_adapt_exact(Nt, Nc, Nk, Na, Nl, mode):
    """Whole numbers; A has few entries a row, so that every value of the low
    rank product has at most 16 bits (two parts in bf16) and no sum passes 2^24."""
    say(f"[adapt exact] {Nt} {Nc} {Nk} {Na} {Nl} {mode}")
    ti, to = TYPES[mode]
    gen = torch.Generator().manual_seed(Nt + Nc)
    In, Ker = _whole(gen, Nt, Nc, dtype=ti), _whole(gen, Nk, Nc, dtype=ti)
    A, B = _whole(gen, Na, Nl, Nc, top=1, dtype=ti), _whole(gen, Na, Nk, Nl, top=1, dtype=ti)
    scales = 2.0 ** torch.randint(-1, 2, (Na,), generator=gen)
    ids = torch.randint(-2, Na + 2, (Nt,), generator=gen).int()
    want = In.float() @ Ker.float().t()
    for a in range(Na):
        at = ids == a
        want[at] += scales[a] * (In[at].float() @ A[a].float().t()) @ B[a].float().t()
    out = torch.full((Nt, Nk), float("nan"), dtype=to, device="cuda")
    i, k, a, b = In.cuda(), Ker.cuda(), A.cuda(), B.cuda()
    ws = routed.adapt_workspace(i, k, a, out)
    routed.adapt_fwd(i, k, a, b, ids.cuda(), out, scales.cuda(), ws)
    assert torch.equal(out.cpu(), want.to(to))
