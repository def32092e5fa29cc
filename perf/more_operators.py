"""The work that the speed of the balance losses and of the 4-bit contractions is
measured on.

Every case is one pass through operators of ``paper_2105_13480_amd.routed`` as
a program that trains or serves routed layers calls them, or the same
operators in elementary torch operations in 32 bits (``own`` false):

* ``"balance"``  a router's per-expert counts, its balance loss and its loss on
  the size of the logits, and their gradient;
* ``"quant"``    values to 4 bits with a shared scale for every 32, and back;
* ``"fwd4"``     the experts' products on gathered rows, Ker in 4 bits;
* ``"fwd44"``    the rows to 4 bits first, then the products of both in 4 bits;
* ``"bwd4"``     the gradient of In, Ker in 4 bits.

4 bits: a block of 32 consecutive values of a row has one scale byte s, 2^(s -
127), and each value is sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 times that.
Two values a byte, the first in the low half; rows are whole blocks, zeros past
their end.

Sizes: Nt rows (tokens), Ng groups (experts), Kt experts of a row, Ns
sequences, Nc input and Nk output features.

``python3 perf/more_operators.py`` lists the cases.
"""
from __future__ import annotations

import math

import torch

own = False


# ---- cases ------------------------------------------------------------------

def listed():
    return [
        # The router of one small training batch: the smallest call, where the
        # launches count.
        {"name": "balance_small", "op": "balance", "ltype": "f32", "olt": "f32", "Nt": 256, "Ng": 32, "Kt": 4,
         "Ns": 1, "pad": 0.0},
        # Sequences of many lengths packed into one training batch, padded at
        # its end, over many experts.
        {"name": "balance_packed", "op": "balance", "ltype": "bf16", "olt": "bf16", "Nt": 16384, "Ng": 128, "Kt": 8,
         "Ns": 37, "pad": 0.06},
        # The rows of a middling batch on their way into a 4-bit product, an odd
        # number of them.
        {"name": "quant_rows", "op": "quant", "itype": "bf16", "otype": "bf16", "Nt": 1001, "Nc": 2048,
         "rule": "floor"},
        # An optimiser's fp32 weights to 4 bits, as a layer is prepared for
        # serving.
        {"name": "quant_weights", "op": "quant", "itype": "f32", "otype": "bf16", "Nt": 32768, "Nc": 2048,
         "rule": "up"},
        # One decoding step of eight requests: the chosen experts' weights are
        # nearly all of the traffic.
        {"name": "fwd4_step", "op": "fwd4", "otype": "f32", "Nt": 8, "Ng": 32, "active": 20, "Kt": 4, "drop": 0.0,
         "Nc": 2048, "Nk": 1024},
        # A middling batch: some rows for each expert, some experts idle, some
        # rows dropped.
        {"name": "fwd4_batch", "op": "fwd4", "otype": "bf16", "Nt": 256, "Ng": 32, "active": 28, "Kt": 2,
         "drop": 0.05, "Nc": 1024, "Nk": 4096},
        # A large prompt batch with 4-bit weights and bf16 rows (the largest case).
        {"name": "fwd4_prompt", "op": "fwd4", "otype": "bf16", "Nt": 16384, "Ng": 16, "active": 16, "Kt": 2,
         "drop": 0.0, "Nc": 2048, "Nk": 4096},
        # Odd sizes throughout: rows that end inside a block.
        {"name": "fwd4_odd", "op": "fwd4", "otype": "f32", "Nt": 1501, "Ng": 7, "active": 6, "Kt": 2, "drop": 0.0,
         "Nc": 515, "Nk": 771},
        # A batch of requests with both sides in 4 bits: the weights' bytes again,
        # and the rows' quantisation before.
        {"name": "fwd44_batch", "op": "fwd44", "otype": "bf16", "Nt": 384, "Ng": 64, "active": 60, "Kt": 4,
         "drop": 0.0, "Nc": 2048, "Nk": 1536},
        # A large prompt batch with both sides in 4 bits: the matrix unit at its
        # highest rate.
        {"name": "fwd44_prompt", "op": "fwd44", "otype": "bf16", "Nt": 16384, "Ng": 16, "active": 16, "Kt": 2,
         "drop": 0.0, "Nc": 2048, "Nk": 4096},
        # A training step through frozen 4-bit experts: the gradient on its way to
        # the adapters below.
        {"name": "bwd4_train", "op": "bwd4", "otype": "bf16", "Nt": 8192, "Ng": 8, "active": 8, "Kt": 2,
         "drop": 0.05, "Nc": 2048, "Nk": 2048},
        # The same of a small batch and odd sizes.
        {"name": "bwd4_odd", "op": "bwd4", "otype": "f32", "Nt": 333, "Ng": 12, "active": 11, "Kt": 2, "drop": 0.0,
         "Nc": 1001, "Nk": 1537},
    ]


def _log(rng, lo, hi):
    """A whole number spread evenly over the logarithm of [lo, hi]."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _rows(rng, hi):
    """A number of rows: a few, a power of two, or what happens to come
    together (odd)."""
    n = _log(rng, 1, hi)
    return n if n < 64 else 1 << (n.bit_length() - 1) if rng.random() < 0.5 else min(n | 1, hi)


_WIDTHS = (64, 96, 128, 192, 256, 320, 384, 512, 640, 768, 896, 1024, 1280, 1536, 1792, 2048, 2560, 3584, 4096)


def _features(rng, lo, hi):
    """A feature count: mostly a usual width, else an odd multiple of 8 or an
    odd number."""
    kind = rng.random()
    if kind < 0.6:
        return rng.choice([w for w in _WIDTHS if lo <= w <= hi])
    n = _log(rng, lo, hi)
    return min(n // 16 * 16 + 8, hi) if kind < 0.8 else min(n | 1, hi)


def _draw_balance(rng):
    Ng = _log(rng, 4, 256)
    ltype, olt = rng.choice((("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")))
    Nt = _rows(rng, 16384)
    return {"op": "balance", "ltype": ltype, "olt": olt, "Nt": Nt, "Ng": Ng, "Kt": rng.randint(1, min(8, Ng)),
            "Ns": 1 if rng.random() < 0.3 else _log(rng, 1, min(Nt, 64)), "pad": rng.choice((0.0, 0.0, 0.05, 0.3))}


def _draw_quant(rng):
    return {"op": "quant", "itype": rng.choice(("f32", "bf16", "bf16")), "otype": rng.choice(("f32", "bf16", "bf16")),
            "Nt": _rows(rng, 32768), "Nc": _features(rng, 32, 2048), "rule": rng.choice(("floor", "up"))}


def _draw_group(rng):
    Ng = _log(rng, 1, 64)
    active = rng.randint(max(1, Ng // 2), Ng)
    case = {"op": rng.choice(("fwd4", "fwd4", "fwd44", "fwd44", "bwd4")), "otype": rng.choice(("f32", "bf16", "bf16")),
            "Nt": _rows(rng, 16384), "Ng": Ng, "active": active, "Kt": rng.randint(1, min(4, active)),
            "drop": rng.choice((0.0, 0.0, 0.05, 0.3)), "Nc": _features(rng, 64, 4096),
            "Nk": _features(rng, 64, 4096)}
    case["active"] = min(active, case["Nt"] * case["Kt"])
    return case


# What a drawn case may cost at most: the operations and bytes of the largest
# listed ones.
_MAX_FLOPS, _MAX_BYTES = 5.4e11, 6e8


def draw(rng):
    """One more case: a pass of one of the kinds listed above."""
    case = rng.choice((_draw_balance, _draw_quant, _draw_group, _draw_group, _draw_group))(rng)
    while True:
        w = work(case)
        if w["flops"] <= _MAX_FLOPS and w["bytes"] <= _MAX_BYTES:
            return case
        # too large: fewer rows, then fewer groups
        if case["Nt"] > 64:
            case["Nt"] = case["Nt"] // 2 | case["Nt"] & 1
        else:
            case["Ng"] = max(case["Kt"], case["Ng"] * 3 // 4)
        if "active" in case:
            case["active"] = min(case["active"], case["Ng"], case["Nt"] * case["Kt"])
            case["Kt"] = min(case["Kt"], case["active"])


# ---- inputs -----------------------------------------------------------------

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _blocks(n):
    return -(-n // 32)


def _randn(gen, *shape, scale=1.0, dtype=torch.float32):
    """Normal values, made in pieces of the first axis and rounded at once."""
    out = torch.empty(shape, dtype=dtype, device="cuda")
    step = max(1, (1 << 26) // max(1, out[0].numel()))
    for i in range(0, shape[0], step):
        out[i:i + step] = torch.randn((min(step, shape[0] - i), *shape[1:]), device="cuda", generator=gen) * scale
    return out


def _activations(gen, Nt, Nc, dtype):
    """Rows of a layer: normal values, some features ten times as large, a few
    values that stand out, and rows without anything (padding)."""
    x = torch.randn((Nt, Nc), device="cuda", generator=gen)
    x *= torch.where(torch.rand((1, Nc), device="cuda", generator=gen) < 0.01, 10.0, 1.0)
    x *= torch.where(torch.rand((Nt, Nc), device="cuda", generator=gen) < 0.001, 30.0, 1.0)
    x *= torch.where(torch.rand((Nt, 1), device="cuda", generator=gen) < 0.01, 0.0, 1.0)
    return x.to(dtype)


def _weights4(gen, Ng, Nk, Nc):
    """Trained weights in 4 bits: normal values, rows of different sizes."""
    codes = torch.empty((Ng, Nk, 16 * _blocks(Nc)), dtype=torch.uint8, device="cuda")
    scales = torch.empty((Ng, Nk, _blocks(Nc)), dtype=torch.uint8, device="cuda")
    for g in range(Ng):
        w = torch.randn((Nk, Nc), device="cuda", generator=gen) * Nc ** -0.5
        w *= 0.5 + torch.rand((Nk, 1), device="cuda", generator=gen)
        codes[g], scales[g] = _to_blocks(w, "floor")
    return codes, scales


def _logits(gen, Nt, Ng, dtype):
    """Router outputs: some experts more popular than others, one row in
    sixteen barred from about half of its experts (-inf), one in 64 from some
    by the type's lowest value, one in 256 from all."""
    x = torch.randn((Nt, Ng), device="cuda", generator=gen) * 1.5 + \
        torch.randn((1, Ng), device="cuda", generator=gen) * 0.5
    x = x.to(dtype)
    half = torch.rand((Nt, Ng), device="cuda", generator=gen) < 0.5
    kind = torch.randint(0, 256, (Nt, 1), device="cuda", generator=gen)
    x = torch.where(half & (kind < 16), torch.full_like(x, -math.inf), x)
    x = torch.where(half & (kind >= 16) & (kind < 20), torch.full_like(x, torch.finfo(dtype).min), x)
    # a row with nothing but lowest values has logits of no size to speak of in a
    # loss on their squares: its first expert stays as it was
    x[:, 0] = torch.where(kind[:, 0] < 20, torch.zeros_like(x[:, 0]), x[:, 0])
    return torch.where(kind == 255, torch.full_like(x, -math.inf), x)


def _chosen(logits, Kt):
    """The Kt largest allowed logits of each row, -1 where there are fewer."""
    value, index = torch.sort(logits.float(), dim=1, descending=True, stable=True)
    value, index = value[:, :Kt], index[:, :Kt]
    return torch.where(value > -math.inf, index, torch.full_like(index, -1)).to(torch.int32).contiguous()


def _sequences(gen, case):
    """Starts of Ns sequences of many lengths (some may be empty); the rows past
    the last are padding."""
    Nt, Ns = case["Nt"], case["Ns"]
    end = Nt - int(case["pad"] * Nt)
    cut = torch.sort((torch.rand(Ns - 1, device="cuda", generator=gen) * (end + 1)).long().clamp(0, end)).values
    one = torch.zeros(1, dtype=torch.long, device="cuda")
    return torch.cat([one, cut, one + end]).to(torch.int32)


def _dropped(case):
    """Rows that no expert takes (over capacity): an exact number."""
    lead = -(-case["active"] // case["Kt"])
    return min(int(case["drop"] * case["Nt"]), max(0, case["Nt"] - lead))


def _choice(gen, case):
    """Experts of each row: ``active`` of the Ng are in use, each by at least
    one row, the rest of the rows prefer some; dropped rows have none."""
    Nt, Kt, active = case["Nt"], case["Kt"], case["active"]
    used = torch.randperm(case["Ng"], device="cuda", generator=gen)[:active]
    score = torch.randn((Nt, active), device="cuda", generator=gen) + \
        torch.randn((1, active), device="cuda", generator=gen) * 0.5
    pick = torch.argsort(score, dim=1, descending=True)[:, :Kt]
    lead = -(-active // Kt)
    pick[:lead] = (torch.arange(lead * Kt, device="cuda") % active).reshape(lead, Kt)
    choice = used[pick].to(torch.int32)
    n = _dropped(case)
    if n:
        choice[Nt - n:] = -1
        choice = choice[torch.randperm(Nt, device="cuda", generator=gen)]
    return choice.contiguous()


def _order(choice, Ng):
    """Offsets and rows of the (row, choice) pairs in the order of their
    experts, and of the rows within one."""
    Kt = choice.shape[1]
    flat = choice.reshape(-1).long()
    flat = torch.where(flat < 0, torch.full_like(flat, Ng), flat)
    order = torch.sort(flat, stable=True).indices
    offsets = torch.searchsorted(flat[order], torch.arange(Ng + 1, device=flat.device)).to(torch.int32)
    rows = torch.where(flat[order] < Ng, order // Kt, torch.full_like(order, -1)).to(torch.int32)
    return offsets, rows


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op, Nt = case["op"], case["Nt"]
    if op == "balance":
        logits = _logits(gen, Nt, case["Ng"], _TYPES[case["ltype"]])
        return {"Logits": logits, "choice": _chosen(logits, case["Kt"]), "bounds": _sequences(gen, case),
                "dLoss": torch.rand(2, device="cuda", generator=gen) * torch.tensor([1e-2, 1e-3], device="cuda")}
    if op == "quant":
        return {"In": _activations(gen, Nt, case["Nc"], _TYPES[case["itype"]])}
    Ng, Nc, Nk = case["Ng"], case["Nc"], case["Nk"]
    offsets, rows = _order(_choice(gen, case), Ng)
    x = {"offsets": offsets, "rows": rows}
    if op == "bwd4":
        x["dOut"] = _randn(gen, Nt * case["Kt"], Nk, dtype=torch.bfloat16)
    else:
        x["In"] = _activations(gen, Nt, Nc, torch.bfloat16)
    x["Ker"], x["KerScales"] = _weights4(gen, Ng, Nk, Nc)
    return x


def _new(*shape, dtype):
    return torch.empty(shape, dtype=dtype, device="cuda")


def prepare(case, seed):
    """The inputs, and the buffers that a program keeps: results, workspaces and
    (plain form) the group sizes on the host."""
    s = _inputs(case, seed)
    s["case"] = case
    op, Nt = case["op"], case["Nt"]
    if op == "balance":
        Ng, Ns = case["Ng"], case["Ns"]
        s.update(counts=_new(Ns, Ng, dtype=torch.int32), tokens=_new(Ns, dtype=torch.int32),
                 loss=_new(2, dtype=torch.float32), dLogits=_new(Nt, Ng, dtype=_TYPES[case["olt"]]))
        if own:
            from paper_2105_13480_amd import routed
            s["ws"] = routed.balance_workspace(Nt, Ng, Ns)
        return s
    to = _TYPES[case["otype"]]
    if op in ("quant", "fwd44"):
        s.update(codes=_new(Nt, 16 * _blocks(case["Nc"]), dtype=torch.uint8),
                 scales=_new(Nt, _blocks(case["Nc"]), dtype=torch.uint8))
    if op == "quant":
        s["Out"] = _new(Nt, case["Nc"], dtype=to)
        return s
    s["Out"] = _new(Nt * case["Kt"], case["Nc" if op == "bwd4" else "Nk"], dtype=to)
    s["most"] = int(s["offsets"].diff().max())
    return s


# ---- one pass ---------------------------------------------------------------

def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    from paper_2105_13480_amd import routed
    op = s["case"]["op"]
    if op == "balance":
        routed.balance(s["Logits"], s["choice"], s["counts"], s["tokens"], s["loss"], s["bounds"], s["ws"])
        routed.balance_bwd(s["Logits"], s["choice"], s["counts"], s["tokens"], s["dLoss"], s["dLogits"], s["bounds"])
        return [s["counts"], s["tokens"], s["loss"], s["dLogits"]]
    if op == "quant":
        routed.quantize4(s["In"], s["codes"], s["scales"], rule=s["case"]["rule"])
        return routed.dequantize4(s["codes"], s["scales"], s["Out"])
    if op == "fwd4":
        return routed.group_fwd4(s["In"], s["Ker"], s["KerScales"], s["Out"], s["offsets"], s["rows"])
    if op == "fwd44":
        routed.quantize4(s["In"], s["codes"], s["scales"])
        return routed.group_fwd4(s["codes"], s["Ker"], s["KerScales"], s["Out"], s["offsets"], s["rows"],
                                 InScales=s["scales"])
    return routed.group_bwd_in4(s["dOut"], s["Ker"], s["KerScales"], s["Out"], s["offsets"])


def _run_plain(s):
    return _PLAIN[s["case"]["op"]](s)


def _plain_balance(s):
    case = s["case"]
    Ng, Ns = case["Ng"], case["Ns"]
    x, choice, bounds = s["Logits"].float(), s["choice"].long(), s["bounds"].long()
    allowed = x > -math.inf
    t = torch.arange(x.shape[0], device="cuda")[:, None]
    inside = (t >= bounds[:-1]) & (t < bounds[1:])  # row, sequence
    some = ((choice >= 0).any(1) & allowed.any(1))[:, None]
    member = (inside & some).float()
    # the softmax over allowed experts
    top = torch.where(allowed, x, torch.full_like(x, -math.inf)).amax(1, keepdim=True)
    top = torch.where(some, top, torch.zeros_like(top))
    e = torch.where(allowed, torch.exp(x - top), torch.zeros_like(x))
    total = e.sum(1, keepdim=True)
    p = torch.where(some, e / total, torch.zeros_like(e))
    lse = torch.where(some, top + torch.log(total), torch.zeros_like(top))
    # counts and means of each sequence
    hit = (choice[:, :, None] == torch.arange(Ng, device="cuda")).sum(1)
    counts = (inside.float().t().contiguous() @ hit.float()).to(torch.int32)
    tokens = member.sum(0)
    whole = counts.sum(1, keepdim=True).clamp_min(1)
    f = counts / whole
    mean = (member.t().contiguous() @ p) / tokens.clamp_min(1)[:, None]
    used = (tokens > 0).sum().clamp_min(1)
    rows = tokens.sum().clamp_min(1)
    balance = Ng * (f * mean).sum() / used
    sizes = (member.sum(1, keepdim=True) * lse * lse).sum() / rows
    # the gradient of dLoss . loss
    fr = member @ f
    per = member @ (s["dLoss"][0] * Ng / (used * tokens.clamp_min(1)))[:, None]
    dl = per * p * (fr - (p * fr).sum(1, keepdim=True))
    dl = dl + member.sum(1, keepdim=True) * (s["dLoss"][1] * 2 / rows) * lse * p
    return [counts, tokens.to(torch.int32), torch.stack([balance, sizes]), dl.to(s["dLogits"].dtype)]


def _to_blocks(x, rule):
    """Codes and scales of the rows of x [.., Nc]: fp32, exact but for the
    rounding to 4 bits (to nearest, ties to the even code)."""
    Nc, Nb = x.shape[-1], _blocks(x.shape[-1])
    y = torch.zeros((*x.shape[:-1], 32 * Nb), device="cuda")
    y[..., :Nc] = x
    y = y.reshape(*x.shape[:-1], Nb, 32)
    a = y.abs()
    bits = a.amax(-1, keepdim=True).view(torch.int32)
    # the largest value is below 8 (floor) or at most 6 (up) times the scale
    s = (bits >> 23) - 2
    if rule == "up":
        s = s + ((bits & 0x7fffff) > 0x400000).int()
    s = s.clamp_min(0)
    a = a * ((254 - s) << 23).view(torch.float32)
    code = ((a > 0.25).byte() + (a >= 0.75).byte() + (a > 1.25).byte() + (a >= 1.75).byte() + (a > 2.5).byte() +
            (a >= 3.5).byte() + (a > 5.0).byte())
    bad = bits >= 0x7f800000  # a block that holds an infinity or NaN is NaN
    code = torch.where(bad, torch.zeros_like(code), code + 8 * (y < 0).byte()).reshape(*x.shape[:-1], 16 * Nb, 2)
    s = torch.where(bad, torch.full_like(s, 255), s).byte()
    return code[..., 0] + 16 * code[..., 1], s[..., 0]


def _of_blocks(codes, scales, Nc):
    """The values in fp32."""
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device="cuda")
    table = torch.cat([table, -table])
    c = torch.stack([codes & 15, codes >> 4], -1).reshape(*scales.shape, 32)
    s = scales.int()
    s = torch.where(s == 255, 0x7fc00000, torch.where(s == 0, 0x400000, s << 23)).view(torch.float32)
    return (table[c.int()] * s[..., None]).reshape(*scales.shape[:-1], -1)[..., :Nc]


def _plain_quant(s):
    codes, scales = _to_blocks(s["In"].float(), s["case"]["rule"])
    return _of_blocks(codes, scales, s["case"]["Nc"]).to(s["Out"].dtype)


def _grouped(s, places, product):
    """The product of each group's places, all groups padded to the most rows of
    one: places [Np, K] to [Ng, K, most], and [Ng, M, most] back to [Np, M]."""
    off, most = s["offsets"].long(), s["most"]
    Np = s["Out"].shape[0]
    at = off[:-1, None] + torch.arange(most, device="cuda")
    part = places[at.clamp_max(Np - 1)].transpose(1, 2).contiguous()
    r = product(part).transpose(1, 2)
    p = torch.arange(Np, device="cuda")
    g = torch.searchsorted(off, p, right=True) - 1
    taken = p < off[-1]
    g = torch.where(taken, g, torch.zeros_like(g))
    out = r[g, torch.where(taken, p - off[g], torch.zeros_like(p))]
    return torch.where(taken[:, None], out, torch.zeros_like(out)).to(s["Out"].dtype)


def _plain_fwd4(s):
    ker = _of_blocks(s["Ker"], s["KerScales"], s["case"]["Nc"])
    return _grouped(s, s["In"].float()[s["rows"].long().clamp_min(0)], lambda x: torch.bmm(ker, x))


def _plain_fwd44(s):
    Nc = s["case"]["Nc"]
    ker, rows = _of_blocks(s["Ker"], s["KerScales"], Nc), _of_blocks(*_to_blocks(s["In"].float(), "floor"), Nc)
    return _grouped(s, rows[s["rows"].long().clamp_min(0)], lambda x: torch.bmm(ker, x))


def _plain_bwd4(s):
    ker = _of_blocks(s["Ker"], s["KerScales"], s["case"]["Nc"]).transpose(1, 2).contiguous()
    return _grouped(s, s["dOut"].float(), lambda x: torch.bmm(ker, x))


_PLAIN = {"balance": _plain_balance, "quant": _plain_quant, "fwd4": _plain_fwd4, "fwd44": _plain_fwd44,
          "bwd4": _plain_bwd4}


# ---- what a pass cannot do without --------------------------------------------

def work(case):
    """Each input that some result needs read once, each result written once."""
    op, Nt = case["op"], case["Nt"]
    size = {"f32": 4, "bf16": 2}
    if op == "balance":
        Ng, Ns = case["Ng"], case["Ns"]
        return {"bytes": Nt * Ng * (size[case["ltype"]] + size[case["olt"]]) + 4 * Nt * case["Kt"] + 4 * Ns * Ng,
                "flops": 16 * Nt * Ng}
    Nc = case["Nc"]
    eo = size[case["otype"]]
    if op == "quant":
        return {"bytes": Nt * (Nc * (size[case["itype"]] + eo) + 17 * _blocks(Nc)), "flops": 8 * Nt * Nc}
    Nk, Np = case["Nk"], Nt * case["Kt"]
    P = (Nt - _dropped(case)) * case["Kt"]
    ker = 17 * case["active"] * Nk * _blocks(Nc)
    if op == "bwd4":
        return {"bytes": 2 * P * Nk + ker + eo * Np * Nc, "flops": 2 * P * Nc * Nk}
    return {"bytes": 2 * min(Nt, P) * Nc + ker + eo * Np * Nk + 4 * Np, "flops": 2 * P * Nc * Nk}


# ---- the definition in 64 bits ------------------------------------------------

def exact(case, seed):
    return _EXACT[case["op"]](case, _inputs(case, seed))


def _exact_balance(case, x):
    """Sequence by sequence, with the gradient by automatic differentiation."""
    Ng, Ns = case["Ng"], case["Ns"]
    logits = x["Logits"].double().cpu()
    choice, bounds = x["choice"].long().cpu(), x["bounds"].tolist()
    leaf = logits.clone().requires_grad_()
    counts = torch.zeros((Ns, Ng), dtype=torch.int32)
    tokens = torch.zeros(Ns, dtype=torch.int32)
    balance, squares = torch.zeros((), dtype=torch.float64), torch.zeros((), dtype=torch.float64)
    for s in range(Ns):
        rows = torch.arange(bounds[s], bounds[s + 1])
        picked = choice[rows].reshape(-1)
        counts[s] = torch.bincount(picked[picked >= 0], minlength=Ng).int()
        rows = rows[(choice[rows] >= 0).any(1) & (logits[rows] > -math.inf).any(1)]
        tokens[s] = rows.numel()
        if rows.numel():
            lse = torch.logsumexp(leaf[rows], 1)
            share = counts[s].double() / counts[s].sum()
            balance = balance + Ng * (share * torch.softmax(leaf[rows], 1).mean(0)).sum()
            squares = squares + (lse * lse).sum()
    loss = torch.stack([balance / max(1, int((tokens > 0).sum())), squares / max(1, int(tokens.sum()))])
    if loss.requires_grad:
        (loss * x["dLoss"].double().cpu()).sum().backward()
    grad = torch.zeros_like(logits) if leaf.grad is None else leaf.grad
    return [counts.cuda(), tokens.cuda(), loss.detach().cuda(), grad.cuda()]


def _exact_blocks(x, rule):
    """The values that the rows of x [Nt, Nc] are rounded to: the nearest of the
    sixteen multiples of each block's scale."""
    Nt, Nc = x.shape
    out = torch.empty((Nt, Nc), dtype=torch.float64, device="cuda")
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device="cuda")
    for c in range(0, Nc, 32):
        v = x[:, c:c + 32].double()
        top = v.abs().amax(1, keepdim=True)
        mantissa, exponent = torch.frexp(top)  # in [1/2, 1)
        e = exponent - 3
        if rule == "up":
            e = torch.where(mantissa > 0.75, e + 1, e)
        e = torch.where(top == 0, torch.full_like(e, -127), e).clamp_min(-127)
        unit = torch.ldexp(torch.ones_like(top), e)
        away = (v.abs()[..., None] - unit[..., None] * table).abs()
        least = away.amin(-1, keepdim=True)
        near = away == least  # two where it is a tie
        low = near.int().argmax(-1)
        high = 7 - near.flip(-1).int().argmax(-1)
        pick = torch.where(low % 2 == 0, low, high)
        out[:, c:c + 32] = torch.sign(v) * table[pick] * unit
    return out


def _exact_quant(case, x):
    if case["Nt"] * case["Nc"] > 1 << 27:
        return None
    out = torch.empty((case["Nt"], case["Nc"]), dtype=torch.float64, device="cuda")
    for t in range(0, case["Nt"], 4096):
        out[t:t + 4096] = _exact_blocks(x["In"][t:t + 4096], case["rule"])
    return out


def _exact_values(codes, scales, Nc):
    """The values of one matrix in 4 bits, byte by byte."""
    out = torch.empty((codes.shape[0], 2 * codes.shape[1]), dtype=torch.float64, device="cuda")
    for half in (0, 1):
        c = (codes.int() // 16 ** half) % 16
        m, e, sign = c % 2, c // 2 % 4, 1 - 2 * (c // 8)
        size = torch.where(e == 0, 0.5 * m.double(), (1 + 0.5 * m.double()) * torch.ldexp(torch.ones_like(m).double(), e - 1))
        out[:, half::2] = sign * size
    unit = torch.ldexp(torch.ones(scales.shape, dtype=torch.float64, device="cuda"), scales.int() - 127)
    unit[scales == 255] = math.nan
    return (out.reshape(*scales.shape, 32) * unit[..., None]).reshape(codes.shape[0], -1)[:, :Nc]


def _exact_group(case, x):
    op, Nc = case["op"], case["Nc"]
    out = torch.zeros((case["Nt"] * case["Kt"], Nc if op == "bwd4" else case["Nk"]), dtype=torch.float64, device="cuda")
    if op == "fwd44":
        rows = torch.cat([_exact_blocks(x["In"][t:t + 4096], "floor") for t in range(0, case["Nt"], 4096)])
    elif op == "fwd4":
        rows = x["In"].double()
    b = x["offsets"].tolist()
    for g in range(case["Ng"]):
        if b[g] < b[g + 1]:
            ker = _exact_values(x["Ker"][g], x["KerScales"][g], Nc)
            if op == "bwd4":
                out[b[g]:b[g + 1]] = torch.mm(x["dOut"][b[g]:b[g + 1]].double(), ker)
            else:
                out[b[g]:b[g + 1]] = torch.mm(rows[x["rows"][b[g]:b[g + 1]].long()], ker.t().contiguous())
    return out


_EXACT = {"balance": _exact_balance, "quant": _exact_quant, "fwd4": _exact_group, "fwd44": _exact_group,
          "bwd4": _exact_group}


if __name__ == "__main__":
    for c in listed():
        w = work(c)
        sizes = {k: v for k, v in c.items() if k not in ("name", "op")}
        print(f"{c['name']:15s} {c['op']:8s} {w['flops'] / 1e9:9.3f} GFLOP {w['bytes'] / 1e6:8.2f} MB  {sizes}")
