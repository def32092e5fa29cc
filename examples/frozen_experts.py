"""A layer of routed experts whose weights are frozen in 4 bits, on one GPU: the
router is trained, with the losses that keep its choices even, and the gradient
goes on through the experts to what is below.

    choice, weights, grouped order = route(logits)                    route
    losses, counts of the choices                                     balance
    x = In in 4 bits;  h = x[rows] K1[e]^T                            quantize4, group_fwd4
    z = relu(h)^2 K2[e]^T                                             group_fwd4
    Out = sum_j weights_j z[slot_j]                                   combine

The gradient of In passes the rounding of its values as it is (straight through).
Python launches only, and nothing waits for the GPU: a step of a fixed size may be
captured into a graph.

    python examples/frozen_experts.py [--rows 4096] [--features 1024] [--steps 20]
"""
import argparse
import os
import sys
import time

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

from paper_2105_13480_amd import routed  # noqa: E402


def in_four_bits(weights, rule="up"):
    """Codes and scales of a tensor of weights."""
    blocks = routed.blocks4(weights.shape[-1])
    new = lambda n: torch.empty((*weights.shape[:-1], n), dtype=torch.uint8, device=weights.device)  # noqa: E731
    return routed.quantize4(weights, new(16 * blocks), new(blocks), rule=rule)


class FrozenExperts:
    """Experts of features x hidden.  Results and gradients bfloat16, logits and
    their gradients float32."""

    def __init__(self, features, hidden, experts, choices, rows, sequences=1, four_bit_rows=True, seed=0):
        gen = torch.Generator().manual_seed(seed)

        def weight(*shape):
            return (torch.randn(shape, generator=gen) / shape[-1] ** 0.5).cuda()

        self.K1, self.K1s = in_four_bits(weight(experts, hidden, features))
        self.K2, self.K2s = in_four_bits(weight(experts, features, hidden))
        self.four_bit_rows = four_bit_rows
        # kept from step to step
        i32 = lambda *s: torch.empty(s, dtype=torch.int32, device="cuda")  # noqa: E731
        u8 = lambda *s: torch.empty(s, dtype=torch.uint8, device="cuda")  # noqa: E731
        blocks = routed.blocks4(features)
        self.order = routed.Routing(rows, experts, choices)
        self.counts, self.tokens, self.losses = i32(sequences, experts), i32(sequences), torch.empty(2, device="cuda")
        self.ws = routed.balance_workspace(rows, experts, sequences)
        self.x, self.xs = u8(rows, 16 * blocks), u8(rows, blocks)

    def _new(self, *shape, dtype=torch.bfloat16):
        return torch.empty(shape, dtype=dtype, device="cuda")

    def forward(self, In, logits, bounds=None):
        """Out [rows, features], the losses (balance, size of the logits) and what
        ``backward`` needs.  bounds: starts of the sequences, None: one."""
        N, C = In.shape
        o = routed.route(logits, self.order, over="all")
        routed.balance(logits, o.choice, self.counts, self.tokens, self.losses, bounds, self.ws)
        Np = o.rows.shape[0]
        h = self._new(Np, self.K1.shape[1])
        if self.four_bit_rows:
            routed.quantize4(In, self.x, self.xs)
            routed.group_fwd4(self.x, self.K1, self.K1s, h, o.offsets, o.rows, InScales=self.xs)
        else:
            routed.group_fwd4(In, self.K1, self.K1s, h, o.offsets, o.rows)
        z = routed.group_fwd4(torch.relu(h).square_(), self.K2, self.K2s, self._new(Np, C), o.offsets)
        return routed.combine(z, self._new(N, C), o.slots, o.gates), self.losses, (logits, bounds, h, z)

    def backward(self, dOut, dLosses, kept):
        """dIn and dLogits, for the order that the last ``forward`` left."""
        logits, bounds, h, z = kept
        N, C = dOut.shape
        o = self.order
        dz, dGates = routed.combine_bwd(dOut, z, torch.empty_like(z), self._new(*o.gates.shape, dtype=torch.float32),
                                        o.slots, o.rows, o.gates)
        dh = routed.group_bwd_in4(dz, self.K2, self.K2s, torch.empty_like(h), o.offsets)
        dh.mul_(torch.relu(h).mul_(2))
        places = routed.group_bwd_in4(dh, self.K1, self.K1s, self._new(h.shape[0], C), o.offsets)
        dIn = routed.combine(places, self._new(N, C), o.slots)  # a row's places add up
        dLogits = routed.route_bwd(logits, o.choice, o.gates, dGates, torch.empty_like(logits), over="all")
        routed.balance_bwd(logits, o.choice, self.counts, self.tokens, dLosses, dLogits, bounds, add=True)
        return dIn, dLogits


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
    for name, value in (("rows", 4096), ("features", 1024), ("hidden", 2048), ("experts", 16), ("choices", 2),
                        ("sequences", 4), ("steps", 20)):
        p.add_argument(f"--{name}", type=int, default=value)
    a = p.parse_args(argv)
    layer = FrozenExperts(a.features, a.hidden, a.experts, a.choices, a.rows, a.sequences)
    gen = torch.Generator().manual_seed(1)
    In = torch.randn((a.rows, a.features), generator=gen).bfloat16().cuda()
    logits = torch.randn((a.rows, a.experts), generator=gen).cuda()
    dOut = torch.randn((a.rows, a.features), generator=gen).bfloat16().cuda()
    dLosses = torch.tensor([1e-2, 1e-3], device="cuda")
    bounds = torch.tensor([a.rows * i // a.sequences for i in range(a.sequences + 1)], dtype=torch.int32, device="cuda")
    forward = _time(lambda: layer.forward(In, logits, bounds), a.steps)
    both = _time(lambda: layer.backward(dOut, dLosses, layer.forward(In, logits, bounds)[2]), a.steps)
    counts = layer.counts.sum(0).tolist()
    print(f"{a.rows} rows, {a.experts} experts of {a.features} x {a.hidden} in 4 bits, {a.choices} a row: "
          f"forward {forward:.3f} ms, with the gradients {both:.3f} ms; choices of an expert {min(counts)} to "
          f"{max(counts)}, balance {layer.losses[0].item():.3f}")


if __name__ == "__main__":
    main()
