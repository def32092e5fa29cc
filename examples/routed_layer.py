"""A layer of routed experts on one GPU, forward and backward, from the
library's routed contractions: an adapted projection, the router, the experts'
two products over the grouped rows, and the weighted return.

    y = In W^T + scales[a] (In A[a]^T) B[a]^T        (a = ids[row])   adapt_fwd
    logits = y R^T                                                    group_fwd, one group
    choice, weights, grouped order                                    route
    h = y[rows] K1[e]^T;  z = relu(h)^2 K2[e]^T                       group_fwd, twice
    Out = sum_j weights_j z[slot_j]                                   combine

Python launches only: nothing waits for the GPU, and the sizes of the groups
stay on it, so that a step of a fixed size may be captured into a graph.

    python examples/routed_layer.py [--rows 4096] [--features 1024] [--steps 20]
"""
import argparse
import os
import sys
import time

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

from paper_2105_13480_amd import routed  # noqa: E402


class RoutedLayer:
    """Weights of one type (float32 or bfloat16); what a step keeps for its
    gradient is float32 or of that type."""

    def __init__(self, features, hidden, experts, choices, adapters, ranks, rows,
                 dtype=torch.bfloat16, over="chosen", seed=0):
        gen = torch.Generator().manual_seed(seed)

        def weight(*shape):
            return (torch.randn(shape, generator=gen) / shape[-1] ** 0.5).to(dtype).cuda()

        self.dtype, self.over, self.rows, self.adapters = dtype, over, rows, adapters
        self.W = weight(features, features)
        self.A = weight(adapters, ranks, features)
        self.B = weight(adapters, features, ranks)
        self.scales = (0.5 + torch.rand(adapters, generator=gen)).cuda()
        self.R = weight(1, experts, features)
        self.K1 = weight(experts, hidden, features)
        self.K2 = weight(experts, features, hidden)
        # kept from step to step: the router's order and its workspace, the
        # adapters' order, the products' workspace, the order of a single group
        self.order = routed.Routing(rows, experts, choices)
        self.by_adapter = routed.Routing(rows, adapters, 1)
        self.one = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
        self.ws = routed.adapt_workspace(self._new(rows, features), self.W, self.A,
                                         self._new(rows, features))

    def _new(self, *shape, dtype=None):
        return torch.empty(shape, dtype=dtype or self.dtype, device="cuda")

    def parameters(self):
        return {"W": self.W, "A": self.A, "B": self.B, "R": self.R, "K1": self.K1, "K2": self.K2}

    def forward(self, In, ids):
        """Out [rows, features] and what ``backward`` needs."""
        N, C = In.shape
        o = self.order
        y = routed.adapt_fwd(In, self.W, self.A, self.B, ids, self._new(N, C), self.scales, self.ws)
        logits = routed.group_fwd(y, self.R, self._new(N, self.R.shape[1], dtype=torch.float32),
                                  self.one)
        routed.route(logits, o, over=self.over)
        Np = o.rows.shape[0]
        h = routed.group_fwd(y, self.K1, self._new(Np, self.K1.shape[1]), o.offsets, o.rows)
        s = torch.relu(h).square_()
        z = routed.group_fwd(s, self.K2, self._new(Np, C), o.offsets)
        Out = routed.combine(z, self._new(N, C), o.slots, o.gates)
        return Out, (In, ids, y, logits, h, s, z)

    def backward(self, dOut, kept):
        """dIn and the gradients of ``parameters()``, of the order and the
        weights that the last ``forward`` left."""
        In, ids, y, logits, h, s, z = kept
        N, C = In.shape
        o, new = self.order, self._new
        grad = {name: torch.empty_like(p) for name, p in self.parameters().items()}
        # the return: every place gets its row's gradient, every choice its weight's
        dz, dGates = routed.combine_bwd(dOut, z, torch.empty_like(z),
                                        new(*o.gates.shape, dtype=torch.float32), o.slots, o.rows,
                                        o.gates)
        # the experts
        routed.group_bwd_ker(dz, s, grad["K2"], o.offsets)
        dh = routed.group_bwd_in(dz, self.K2, torch.empty_like(h), o.offsets)
        dh.mul_(torch.relu(h).mul_(2))
        routed.group_bwd_ker(dh, y, grad["K1"], o.offsets, o.rows)
        dplaces = routed.group_bwd_in(dh, self.K1, new(h.shape[0], C), o.offsets)
        dy = routed.combine(dplaces, new(N, C), o.slots)  # the gather: a row's places add up
        # the router
        dlogits = routed.route_bwd(logits, o.choice, o.gates, dGates, new(*logits.shape, dtype=torch.float32),
                                   over=self.over).to(self.dtype)
        routed.group_bwd_ker(dlogits, y, grad["R"], self.one)
        dy += routed.group_bwd_in(dlogits, self.R, new(N, C), self.one)
        # the adapted projection: rows in the order of their adapters (a choice
        # of one, with no logit but the row's own adapter's)
        allowed = ids[:, None] == torch.arange(self.adapters, dtype=torch.int32, device="cuda")
        b = routed.route(torch.where(allowed, 0.0, -float("inf")), self.by_adapter)
        place = b.rows.clamp(min=0).long()
        scale = self.scales[ids.clamp(0, self.adapters - 1).long()]
        dt = (dy * scale[:, None]).to(self.dtype)[place]  # places without an adapter are in no group
        low = routed.group_fwd(In, self.A, new(N, self.A.shape[1]), b.offsets, b.rows)
        routed.group_bwd_ker(dt, low, grad["B"], b.offsets)
        dlow = routed.group_bwd_in(dt, self.B, torch.empty_like(low), b.offsets)
        routed.group_bwd_ker(dlow, In, grad["A"], b.offsets, b.rows)
        routed.group_bwd_ker(dy, In, grad["W"][None], self.one)
        dIn = routed.combine(routed.group_bwd_in(dlow, self.A, new(N, C), b.offsets), new(N, C), b.slots)
        dIn += routed.group_bwd_in(dy, self.W[None], new(N, C), self.one)
        return dIn, grad


def _time(step, steps):
    for _ in range(3):
        step()
    torch.cuda.synchronize()
    start = time.perf_counter()
    for _ in range(steps):
        step()
    torch.cuda.synchronize()
    return (time.perf_counter() - start) / steps * 1e3


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    for name, value in (("rows", 4096), ("features", 1024), ("hidden", 2048), ("experts", 16),
                        ("choices", 2), ("adapters", 4), ("ranks", 16), ("steps", 20)):
        p.add_argument(f"--{name}", type=int, default=value)
    a = p.parse_args(argv)
    layer = RoutedLayer(a.features, a.hidden, a.experts, a.choices, a.adapters, a.ranks, a.rows)
    gen = torch.Generator().manual_seed(1)
    In = torch.randn((a.rows, a.features), generator=gen).bfloat16().cuda()
    ids = torch.randint(-1, a.adapters, (a.rows,), generator=gen).int().cuda()  # -1: no adapter
    dOut = torch.randn((a.rows, a.features), generator=gen).bfloat16().cuda()
    forward = _time(lambda: layer.forward(In, ids), a.steps)
    both = _time(lambda: layer.backward(dOut, layer.forward(In, ids)[1]), a.steps)
    counts = layer.order.offsets.diff().tolist()
    print(f"{a.rows} rows, {a.experts} experts of {a.features} x {a.hidden}, {a.choices} a row: "
          f"forward {forward:.3f} ms, with the gradients {both:.3f} ms; "
          f"rows of the experts {min(counts)} to {max(counts)}")


if __name__ == "__main__":
    main()
