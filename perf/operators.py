"""The work that the routed contractions' speed is measured on.

Every case is one pass through an operator of ``paper_2105_13480_amd.routed``
as a program that trains or serves routed layers calls it, or the same
operator in elementary torch operations in 32 bits (``own`` false):

* ``"route"``      the experts of each row, their weights and the grouped order;
* ``"combine"``    the weighted return of the experts' rows to their tokens;
* ``"route_bwd"``  both halves' gradients, as a training step calls them in a row;
* ``"group_fwd"``  the experts' products on gathered rows;
* ``"group_bwd"``  their gradients with respect to In and Ker;
* ``"adapt"``      a shared projection with a low-rank adapter for each row.

Types are the library's three: ``f32``, ``bf16`` (fp32 results) and
``bf16_obf16`` (bf16 results).  Sizes: Nt rows (tokens), Ng groups (experts),
Kt experts of a row, Nc input and Nk output features, Na adapters of rank Nl.

``python3 perf/operators.py`` lists the cases.
"""
from __future__ import annotations

import math

import torch

own = False


# ---- cases ------------------------------------------------------------------

def listed():
    return [
        # One decoding step of sixteen requests: the smallest call, where the
        # launches count.
        {"name": "route_step", "op": "route", "Nt": 16, "Ng": 32, "Kt": 4, "ltype": "f32", "over": "chosen"},
        # A long prompt batch over many experts; bf16 logits tie often, and some
        # rows may not use some experts, or any.
        {"name": "route_prompt", "op": "route", "Nt": 16384, "Ng": 128, "Kt": 8, "ltype": "bf16", "over": "all"},
        # The return of a prompt's expert rows to their tokens: pure traffic.
        {"name": "combine_prompt", "op": "combine", "dtype": "bf16_obf16", "Nt": 8192, "Ng": 64, "Kt": 4,
         "drop": 0.0, "Nk": 2048},
        # The gradients of return and router in one training step.
        {"name": "route_train", "op": "route_bwd", "dtype": "bf16_obf16", "ltype": "f32", "over": "all",
         "Nt": 8192, "Ng": 64, "Kt": 2, "drop": 0.05, "Nk": 2048},
        # One decoding step of eight requests: the chosen experts' weights are
        # nearly all of the traffic.
        {"name": "group_step", "op": "group_fwd", "dtype": "bf16", "Nt": 8, "Ng": 32, "active": 20, "Kt": 4,
         "drop": 0.0, "Nc": 2048, "Nk": 1024},
        # A middling batch: a few rows for each expert, some experts idle, some
        # rows dropped.
        {"name": "group_batch", "op": "group_fwd", "dtype": "bf16_obf16", "Nt": 256, "Ng": 32, "active": 28,
         "Kt": 2, "drop": 0.05, "Nc": 1024, "Nk": 4096},
        # A large prompt batch: matrix products throughout (the largest case).
        {"name": "group_prompt", "op": "group_fwd", "dtype": "bf16_obf16", "Nt": 16384, "Ng": 16, "active": 16,
         "Kt": 2, "drop": 0.0, "Nc": 2048, "Nk": 4096},
        # Odd sizes throughout in full precision, as a reference run has them.
        {"name": "group_odd_f32", "op": "group_fwd", "dtype": "f32", "Nt": 1501, "Ng": 7, "active": 6, "Kt": 2,
         "drop": 0.0, "Nc": 515, "Nk": 771},
        # A training step's gradients: both products over the same rows, the
        # weights' gradient in fp32 for the optimiser.
        {"name": "group_train", "op": "group_bwd", "dtype": "bf16", "Nt": 8192, "Ng": 8, "active": 8, "Kt": 2,
         "drop": 0.05, "Nc": 2048, "Nk": 2048},
        # One decoding step of 48 requests, each with an adapter of its own
        # choice or none.
        {"name": "adapt_step", "op": "adapt", "dtype": "bf16_obf16", "Nt": 48, "Nc": 4096, "Nk": 4096, "Na": 24,
         "Nl": 16, "request": 1},
        # Prompts of some hundred rows of many requests packed into one batch.
        {"name": "adapt_prompt", "op": "adapt", "dtype": "bf16_obf16", "Nt": 8192, "Nc": 2048, "Nk": 4096, "Na": 8,
         "Nl": 64, "request": 400},
        # Odd sizes in full precision.
        {"name": "adapt_odd_f32", "op": "adapt", "dtype": "f32", "Nt": 333, "Nc": 1001, "Nk": 1537, "Na": 5,
         "Nl": 12, "request": 30},
    ]


def _log(rng, lo, hi):
    """A whole number spread evenly over the logarithm of [lo, hi]."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _rows(rng, hi):
    """A number of rows: a few, a power of two, or what happens to come
    together (odd)."""
    n = _log(rng, 1, hi)
    return n if n < 64 else 1 << (n.bit_length() - 1) if rng.random() < 0.5 else min(n | 1, hi)


_WIDTHS = (64, 128, 192, 256, 320, 384, 512, 640, 768, 896, 1024, 1280, 1536, 1792, 2048, 2560, 3584, 4096)


def _features(rng, lo, hi):
    """A feature count: mostly a usual width, else an odd multiple of 8 or an
    odd number."""
    kind = rng.random()
    if kind < 0.6:
        return rng.choice([w for w in _WIDTHS if lo <= w <= hi])
    n = _log(rng, lo, hi)
    return min(n // 16 * 16 + 8, hi) if kind < 0.8 else min(n | 1, hi)


def _draw_route(rng):
    Ng = _log(rng, 4, 256)
    return {"op": "route", "Nt": _rows(rng, 16384), "Ng": Ng, "Kt": rng.randint(1, min(8, Ng)),
            "ltype": rng.choice(("f32", "bf16")), "over": rng.choice(("all", "chosen"))}


def _draw_return(rng):
    Ng = _log(rng, 4, 128)
    case = {"op": rng.choice(("combine", "route_bwd")), "dtype": rng.choice(("f32", "bf16", "bf16_obf16")),
            "Nt": _rows(rng, 8192), "Ng": Ng, "Kt": rng.randint(1, min(8, Ng)),
            "drop": rng.choice((0.0, 0.0, 0.05, 0.3)), "Nk": _features(rng, 64, 2048)}
    if case["op"] == "route_bwd":
        case.update(ltype=rng.choice(("f32", "bf16")), over=rng.choice(("all", "chosen")))
    return case


def _draw_group(rng):
    Ng = _log(rng, 2, 64)
    active = rng.randint(max(1, Ng // 2), Ng)
    case = {"op": rng.choice(("group_fwd", "group_fwd", "group_bwd")),
            "dtype": rng.choice(("f32", "bf16", "bf16", "bf16_obf16", "bf16_obf16")),
            "Nt": _rows(rng, 16384), "Ng": Ng, "active": active, "Kt": rng.randint(1, min(4, active)),
            "drop": rng.choice((0.0, 0.0, 0.05, 0.3)), "Nc": _features(rng, 128, 4096),
            "Nk": _features(rng, 128, 4096)}
    case["active"] = min(active, case["Nt"] * case["Kt"])
    return case


def _draw_adapt(rng):
    return {"op": "adapt", "dtype": rng.choice(("f32", "bf16", "bf16_obf16", "bf16_obf16")),
            "Nt": _rows(rng, 8192), "Nc": _features(rng, 256, 4096), "Nk": _features(rng, 256, 4096),
            "Na": _log(rng, 1, 64), "Nl": rng.choice((4, 8, 8, 12, 16, 16, 32, 64)), "request": _log(rng, 1, 1000)}


_DRAWS = (_draw_route, _draw_return, _draw_group, _draw_group, _draw_adapt, _draw_adapt)

# What a drawn case may cost at most: the operations and bytes of the largest
# listed case, and for fp32, whose matrix rate is a sixteenth of bf16's, a
# sixteenth of the operations.
_MAX_FLOPS = {"f32": 3.4e10, "bf16": 5.4e11, "bf16_obf16": 5.4e11}
_MAX_BYTES = 6e8


def draw(rng):
    """One more case: an operator call of one of the kinds listed above."""
    case = rng.choice(_DRAWS)(rng)
    while True:
        w = work(case)
        if w["flops"] <= _MAX_FLOPS[case.get("dtype", "f32")] and w["bytes"] <= _MAX_BYTES:
            return case
        # too large: fewer rows, then fewer groups
        if case["Nt"] > 64:
            case["Nt"] = case["Nt"] // 2 | case["Nt"] & 1
            if "active" in case:
                case["active"] = min(case["active"], case["Nt"] * case["Kt"])
        else:
            case["Ng"] = max(case["Kt"], case["Ng"] * 3 // 4)
            case["active"] = min(case["active"], case["Ng"])
            case["Kt"] = min(case["Kt"], case["active"])


# ---- inputs -----------------------------------------------------------------

_TYPES = {"f32": (torch.float32, torch.float32), "bf16": (torch.bfloat16, torch.float32),
          "bf16_obf16": (torch.bfloat16, torch.bfloat16)}
_LTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _randn(gen, *shape, scale=1.0, dtype=torch.float32):
    """Normal values, made in pieces of the first axis and rounded at once."""
    out = torch.empty(shape, dtype=dtype, device="cuda")
    step = max(1, (1 << 26) // max(1, out[0].numel()))
    for i in range(0, shape[0], step):
        out[i:i + step] = torch.randn((min(step, shape[0] - i), *shape[1:]), device="cuda", generator=gen) * scale
    return out


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
    return torch.where(kind == 255, torch.full_like(x, -math.inf), x)


def _dropped(case):
    """Rows that no expert takes (over capacity): an exact number."""
    lead = -(-case.get("active", 1) // case["Kt"])
    return min(int(case["drop"] * case["Nt"]), max(0, case["Nt"] - lead))


def _choice(gen, case):
    """Experts of each row: ``active`` of the Ng are in use, each by at least
    one row, the rest of the rows prefer some; dropped rows have none."""
    Nt, Ng, Kt = case["Nt"], case["Ng"], case["Kt"]
    active = case.get("active", Ng)
    used = torch.randperm(Ng, device="cuda", generator=gen)[:active]
    score = torch.randn((Nt, active), device="cuda", generator=gen) + \
        torch.randn((1, active), device="cuda", generator=gen) * 0.5
    pick = torch.argsort(score, dim=1, descending=True)[:, :Kt]
    if "active" in case:
        lead = -(-active // Kt)
        first = (torch.arange(lead * Kt, device="cuda") % active).reshape(lead, Kt)
        pick[:lead] = first
    choice = used[pick].to(torch.int32)
    n = _dropped(case)
    if n:
        choice[Nt - n:] = -1
        perm = torch.randperm(Nt, device="cuda", generator=gen)
        choice = choice[perm]
    return choice.contiguous()


def _order(choice, Ng):
    """Offsets, rows and slots of the (row, choice) pairs in the order of their
    experts, and of the rows within one."""
    Nt, Kt = choice.shape
    flat = choice.reshape(-1).long()
    flat = torch.where(flat < 0, torch.full_like(flat, Ng), flat)
    order = torch.sort(flat, stable=True).indices
    experts = torch.arange(Ng + 1, device=flat.device)
    offsets = (flat[:, None] < experts[None, :]).sum(0).to(torch.int32) if flat.numel() * Ng < 1 << 24 else \
        torch.searchsorted(flat[order], experts).to(torch.int32)
    taken = flat[order] < Ng
    rows = torch.where(taken, order // Kt, torch.full_like(order, -1)).to(torch.int32)
    slots = torch.full_like(flat, -1)
    slots[order] = torch.where(taken, torch.arange(order.numel(), device=flat.device), torch.full_like(order, -1))
    return offsets, rows, slots.reshape(Nt, Kt).to(torch.int32)


def _gates(gen, choice):
    g = torch.rand(choice.shape, device="cuda", generator=gen) + 0.1
    g = torch.where(choice < 0, torch.zeros_like(g), g)
    return g / g.sum(1, keepdim=True).clamp_min(1e-6)


def _adapters(gen, case):
    """The adapter of each row: requests of about ``request`` rows in a row,
    one in eight without an adapter."""
    Nt = case["Nt"]
    starts = torch.rand(Nt, device="cuda", generator=gen) < 1.0 / case["request"]
    request = torch.cumsum(starts.long(), 0)
    ids = torch.randint(0, case["Na"], (Nt + 1,), device="cuda", generator=gen)
    none = torch.rand(Nt + 1, device="cuda", generator=gen) < 0.125
    return torch.where(none, torch.full_like(ids, -1), ids)[request].to(torch.int32)


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op, Nt = case["op"], case["Nt"]
    if op == "route":
        return {"Logits": _logits(gen, Nt, case["Ng"], _LTYPES[case["ltype"]])}
    ti, _ = _TYPES[case["dtype"]]
    if op == "adapt":
        Nc, Nk, Na, Nl = case["Nc"], case["Nk"], case["Na"], case["Nl"]
        return {"In": _randn(gen, Nt, Nc, dtype=ti), "Ker": _randn(gen, Nk, Nc, scale=Nc ** -0.5, dtype=ti),
                "A": _randn(gen, Na, Nl, Nc, scale=Nc ** -0.5, dtype=ti),
                "B": _randn(gen, Na, Nk, Nl, scale=0.3 * Nl ** -0.5, dtype=ti), "ids": _adapters(gen, case),
                "scales": torch.rand(Na, device="cuda", generator=gen) + 0.5}
    choice = _choice(gen, case)
    offsets, rows, slots = _order(choice, case["Ng"])
    x = {"choice": choice, "offsets": offsets, "rows": rows, "slots": slots}
    Np = Nt * case["Kt"]
    if op == "combine":
        x.update(In=_randn(gen, Np, case["Nk"], dtype=ti), gates=_gates(gen, choice))
    elif op == "route_bwd":
        logits = (torch.randn((Nt, case["Ng"]), device="cuda", generator=gen) * 1.5).to(_LTYPES[case["ltype"]])
        x.update(In=_randn(gen, Np, case["Nk"], dtype=ti), Logits=logits,
                 dOut=_randn(gen, Nt, case["Nk"], dtype=ti))
        # the weights that the forward pass gave for these choices
        p = torch.softmax(logits.double(), 1)
        g = torch.where(choice < 0, torch.zeros((), dtype=p.dtype, device="cuda"), p.gather(1, choice.clamp_min(0).long()))
        if case["over"] == "chosen":
            g = g / g.sum(1, keepdim=True).clamp_min(1e-300)
        x["gates"] = g.float()
    else:
        Ng, Nc, Nk = case["Ng"], case["Nc"], case["Nk"]
        x["In"] = _randn(gen, Nt, Nc, dtype=ti)
        if op == "group_fwd":
            x["Ker"] = _randn(gen, Ng, Nk, Nc, scale=Nc ** -0.5, dtype=ti)
        else:
            x["Ker"] = _randn(gen, Ng, Nk, Nc, scale=Nk ** -0.5, dtype=ti)
            x["dOut"] = _randn(gen, Np, Nk, dtype=ti)
    return x


def prepare(case, seed):
    """The inputs, and the buffers and handles that a program keeps: results,
    workspaces, and (plain form) the group sizes on the host."""
    state = _inputs(case, seed)
    state["case"] = case
    op, Nt = case["op"], case["Nt"]
    tl = _LTYPES[case.get("ltype", "f32")]
    if op == "route":
        if own:
            from paper_2105_13480_amd import routed
            state["routing"] = routed.Routing(Nt, case["Ng"], case["Kt"])
        return state
    _, to = _TYPES[case["dtype"]]
    if op == "adapt":
        state["Out"] = torch.empty((Nt, case["Nk"]), dtype=to, device="cuda")
        if own:
            from paper_2105_13480_amd import routed
            state["ws"] = routed.adapt_workspace(state["In"], state["Ker"], state["A"], state["Out"])
        else:
            ids = state["ids"]
            state["members"] = [torch.nonzero(ids == a).reshape(-1) for a in range(case["Na"])]
        return state
    Np = Nt * case["Kt"]
    if op == "combine":
        state["Out"] = torch.empty((Nt, case["Nk"]), dtype=to, device="cuda")
    elif op == "route_bwd":
        state["dIn"] = torch.empty((Np, case["Nk"]), dtype=to, device="cuda")
        state["dGates"] = torch.empty((Nt, case["Kt"]), device="cuda")
        state["dLogits"] = torch.empty((Nt, case["Ng"]), dtype=tl, device="cuda")
    elif op == "group_fwd":
        state["Out"] = torch.empty((Np, case["Nk"]), dtype=to, device="cuda")
    else:
        state["dIn"] = torch.empty((Np, case["Nc"]), dtype=to, device="cuda")
        state["dKer"] = torch.empty((case["Ng"], case["Nk"], case["Nc"]), dtype=to, device="cuda")
    if not own:
        state["bounds"] = state["offsets"].tolist()
    return state


# ---- one pass ---------------------------------------------------------------

def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    from paper_2105_13480_amd import routed
    case = s["case"]
    op = case["op"]
    if op == "route":
        r = routed.route(s["Logits"], s["routing"], over=case["over"])
        return [r.choice, r.gates, r.offsets, r.rows, r.slots]
    if op == "combine":
        return routed.combine(s["In"], s["Out"], s["slots"], s["gates"])
    if op == "route_bwd":
        routed.combine_bwd(s["dOut"], s["In"], s["dIn"], s["dGates"], s["slots"], s["rows"], s["gates"])
        routed.route_bwd(s["Logits"], s["choice"], s["gates"], s["dGates"], s["dLogits"], over=case["over"])
        return [s["dIn"], s["dGates"], s["dLogits"]]
    if op == "group_fwd":
        return routed.group_fwd(s["In"], s["Ker"], s["Out"], s["offsets"], s["rows"])
    if op == "group_bwd":
        routed.group_bwd_in(s["dOut"], s["Ker"], s["dIn"], s["offsets"])
        routed.group_bwd_ker(s["dOut"], s["In"], s["dKer"], s["offsets"], s["rows"])
        return [s["dIn"], s["dKer"]]
    return routed.adapt_fwd(s["In"], s["Ker"], s["A"], s["B"], s["ids"], s["Out"], s["scales"], s["ws"])


def _run_plain(s):
    return _PLAIN[s["case"]["op"]](s)


def _plain_route(s):
    case = s["case"]
    x = s["Logits"].float()
    allowed = x > -math.inf
    x = torch.where(allowed, x, torch.full_like(x, -math.inf))
    value, index = torch.sort(x, dim=1, descending=True, stable=True)
    value, index = value[:, :case["Kt"]], index[:, :case["Kt"]]
    taken = value > -math.inf
    top = torch.where(taken[:, :1], value[:, :1], torch.zeros_like(value[:, :1]))
    e = torch.exp(value - top)
    total = (torch.exp(x - top) if case["over"] == "all" else e).sum(1, keepdim=True)
    gates = torch.where(taken, e / total, torch.zeros_like(e))
    choice = torch.where(taken, index, torch.full_like(index, -1)).to(torch.int32)
    return [choice, gates, *_order(choice, case["Ng"])]


def _plain_combine(s):
    slots = s["slots"].long()
    out = torch.zeros(s["Out"].shape, device="cuda")
    for j in range(slots.shape[1]):
        taken = slots[:, j] >= 0
        row = s["In"][slots[:, j].clamp_min(0)].float() * s["gates"][:, j, None]
        out += torch.where(taken[:, None], row, torch.zeros_like(row))
    return out.to(s["Out"].dtype)


def _plain_route_bwd(s):
    case = s["case"]
    slots, dout = s["slots"].long(), s["dOut"].float()
    din = torch.zeros(s["dIn"].shape, device="cuda")
    dgates = torch.zeros(s["dGates"].shape, device="cuda")
    for j in range(slots.shape[1]):
        taken = slots[:, j] >= 0
        at = slots[:, j].clamp_min(0)
        dgates[:, j] = torch.where(taken, (dout * s["In"][at].float()).sum(1), torch.zeros_like(dgates[:, j]))
        # a row without a slot adds zeros to row 0
        part = dout * s["gates"][:, j, None]
        din.index_add_(0, at, torch.where(taken[:, None], part, torch.zeros_like(part)))
    choice = s["choice"].long()
    taken = choice >= 0
    inner = (s["gates"] * dgates).sum(1, keepdim=True)
    dl = torch.zeros(s["dLogits"].shape, device="cuda")
    if case["over"] == "all":
        x = s["Logits"].float()
        p = torch.exp(x - x.amax(1, keepdim=True))
        dl -= p / p.sum(1, keepdim=True) * inner
        dl *= taken.any(1, keepdim=True)
        add = s["gates"] * dgates
    else:
        add = s["gates"] * (dgates - inner)
    dl.scatter_add_(1, choice.clamp_min(0), torch.where(taken, add, torch.zeros_like(add)))
    return [din.to(s["dIn"].dtype), dgates, dl.to(s["dLogits"].dtype)]


def _plain_group_fwd(s):
    b = s["bounds"]
    out = torch.zeros(s["Out"].shape, device="cuda")
    for g in range(len(b) - 1):
        if b[g] < b[g + 1]:
            out[b[g]:b[g + 1]] = s["In"][s["rows"][b[g]:b[g + 1]].long()].float() @ s["Ker"][g].float().t()
    return out.to(s["Out"].dtype)


def _plain_group_bwd(s):
    b = s["bounds"]
    din = torch.zeros(s["dIn"].shape, device="cuda")
    dker = torch.zeros(s["dKer"].shape, device="cuda")
    for g in range(len(b) - 1):
        if b[g] < b[g + 1]:
            dout = s["dOut"][b[g]:b[g + 1]].float()
            din[b[g]:b[g + 1]] = dout @ s["Ker"][g].float()
            dker[g] = dout.t() @ s["In"][s["rows"][b[g]:b[g + 1]].long()].float()
    return [din.to(s["dIn"].dtype), dker.to(s["dKer"].dtype)]


def _plain_adapt(s):
    out = s["In"].float() @ s["Ker"].float().t()
    for a, rows in enumerate(s["members"]):
        if rows.numel():
            h = s["In"][rows].float() @ s["A"][a].float().t()
            out[rows] += s["scales"][a] * (h @ s["B"][a].float().t())
    return out.to(s["Out"].dtype)


_PLAIN = {"route": _plain_route, "combine": _plain_combine, "route_bwd": _plain_route_bwd,
          "group_fwd": _plain_group_fwd, "group_bwd": _plain_group_bwd, "adapt": _plain_adapt}


# ---- what a pass cannot do without --------------------------------------------

def work(case):
    """Each input that some result needs read once, each result written once."""
    op, Nt = case["op"], case["Nt"]
    el = 2 if case.get("ltype") == "bf16" else 4
    if op == "route":
        Ng, pairs = case["Ng"], Nt * case["Kt"]
        return {"bytes": Nt * Ng * el + 16 * pairs + 4 * (Ng + 1), "flops": 4 * Nt * Ng}
    ei = 4 if case["dtype"] == "f32" else 2
    eo = 2 if case["dtype"] == "bf16_obf16" else 4
    if op == "adapt":
        Nc, Nk, Nl = case["Nc"], case["Nk"], case["Nl"]
        # requests with an adapter, and the adapters among Na that they name
        named = max(1.0, Nt / case["request"]) * 0.875
        used = case["Na"] * (1.0 - (1.0 - 1.0 / case["Na"]) ** named)
        return {"bytes": int(ei * (Nt * Nc + Nk * Nc + used * Nl * (Nc + Nk)) + eo * Nt * Nk + 4 * Nt),
                "flops": int(2 * Nt * Nk * Nc + 2 * 0.875 * Nt * Nl * (Nc + Nk))}
    Np = Nt * case["Kt"]
    P = (Nt - _dropped(case)) * case["Kt"]
    if op == "combine":
        Nk = case["Nk"]
        return {"bytes": ei * P * Nk + eo * Nt * Nk + 8 * Np, "flops": 2 * P * Nk}
    if op == "route_bwd":
        Nk, Ng = case["Nk"], case["Ng"]
        return {"bytes": ei * (Nt * Nk + P * Nk) + eo * Np * Nk + 20 * Np + (2 if case["over"] == "all" else 1) * el * Nt * Ng,
                "flops": 3 * P * Nk + 6 * Nt * Ng}
    Nc, Nk, active = case["Nc"], case["Nk"], case["active"]
    if op == "group_fwd":
        return {"bytes": ei * (min(Nt, P) * Nc + active * Nk * Nc) + eo * Np * Nk + 4 * Np, "flops": 2 * P * Nc * Nk}
    return {"bytes": ei * (P * Nk + active * Nk * Nc + min(Nt, P) * Nc) + eo * (Np * Nc + case["Ng"] * Nk * Nc) + 4 * Np,
            "flops": 4 * P * Nc * Nk}


# ---- the definition in 64 bits ------------------------------------------------

def exact(case, seed):
    return _EXACT[case["op"]](case, _inputs(case, seed))


def _exact_route(case, x):
    """One largest allowed logit after the other; the order by counting."""
    Nt, Ng, Kt = case["Nt"], case["Ng"], case["Kt"]
    l = x["Logits"].double().cpu()
    left = torch.where(torch.isnan(l), torch.tensor(-math.inf, dtype=l.dtype), l)
    choice = torch.full((Nt, Kt), -1, dtype=torch.int64)
    value = torch.full((Nt, Kt), -math.inf, dtype=l.dtype)
    column = torch.arange(Ng)
    for j in range(Kt):
        best = left.amax(1)
        first = torch.where(left == best[:, None], column[None, :], Ng).amin(1)
        some = best > -math.inf
        choice[some, j] = first[some]
        value[some, j] = best[some]
        left[some, first[some]] = -math.inf
    top = torch.where(value[:, :1] > -math.inf, value[:, :1], torch.zeros_like(value[:, :1]))
    weight = torch.exp(value - top)
    total = torch.exp(l - top).sum(1, keepdim=True) if case["over"] == "all" else weight.sum(1, keepdim=True)
    gates = torch.where(choice >= 0, weight / torch.where(total > 0, total, torch.ones_like(total)),
                        torch.zeros_like(weight))
    pairs = choice.reshape(-1).numpy()
    lists = [[] for _ in range(Ng)]
    for i, e in enumerate(pairs.tolist()):
        if e >= 0:
            lists[e].append(i)
    offsets = [0]
    for members in lists:
        offsets.append(offsets[-1] + len(members))
    order = torch.tensor([i for members in lists for i in members], dtype=torch.int64)
    rows = torch.full((Nt * Kt,), -1, dtype=torch.int64)
    slots = torch.full((Nt * Kt,), -1, dtype=torch.int64)
    rows[:order.numel()] = order // Kt
    slots[order] = torch.arange(order.numel())
    whole = [torch.tensor(offsets), rows, slots.reshape(Nt, Kt)]
    return [choice.to(torch.int32).cuda(), gates.cuda(), *(t.to(torch.int32).cuda() for t in whole)]


def _exact_combine(case, x):
    """Each grouped row added to the token that it came from."""
    P = int(x["offsets"][-1])
    t = x["rows"][:P].long()
    j = (x["slots"][t] == torch.arange(P, device="cuda")[:, None]).long().argmax(1)
    out = torch.zeros((case["Nt"], case["Nk"]), dtype=torch.float64, device="cuda")
    return out.index_add_(0, t, x["In"][:P].double() * x["gates"][t, j].double()[:, None])


def _exact_route_bwd(case, x):
    P = int(x["offsets"][-1])
    t = x["rows"][:P].long()
    j = (x["slots"][t] == torch.arange(P, device="cuda")[:, None]).long().argmax(1)
    din = torch.zeros(x["In"].shape, dtype=torch.float64, device="cuda")
    dgates = torch.zeros(x["gates"].shape, dtype=torch.float64, device="cuda")
    dout = x["dOut"].double()[t]
    din[:P] = dout * x["gates"][t, j].double()[:, None]
    dgates[t, j] = (dout * x["In"][:P].double()).sum(1)
    # The Jacobian of the softmax, row by row of the choices.
    Nt, Ng = case["Nt"], case["Ng"]
    chosen = torch.zeros((Nt, Ng + 1), dtype=torch.bool, device="cuda")
    spread = torch.zeros((Nt, Ng + 1), dtype=torch.float64, device="cuda")
    at = torch.where(x["choice"] < 0, torch.full_like(x["choice"], Ng), x["choice"]).long()
    chosen.scatter_(1, at, True)
    spread.scatter_(1, at, dgates)
    chosen, spread = chosen[:, :Ng], torch.where(chosen, spread, torch.zeros_like(spread))[:, :Ng]
    l = x["Logits"].double()
    over = torch.ones_like(chosen) if case["over"] == "all" else chosen
    l = torch.where(over, l, torch.full_like(l, -math.inf))
    p = torch.softmax(torch.where(over.any(1, keepdim=True), l, torch.zeros_like(l)), 1)
    dl = p * (spread - (p * spread).sum(1, keepdim=True)) * chosen.any(1, keepdim=True)
    return [din, dgates, dl]


def _exact_group_fwd(case, x):
    out = torch.zeros((case["Nt"] * case["Kt"], case["Nk"]), dtype=torch.float64, device="cuda")
    slots, choice = x["slots"].long(), x["choice"]
    for g in range(case["Ng"]):
        t, j = torch.nonzero(choice == g, as_tuple=True)
        if t.numel():
            out[slots[t, j]] = torch.mm(x["In"][t].double(), x["Ker"][g].double().t().contiguous())
    return out


def _exact_group_bwd(case, x):
    din = torch.zeros((case["Nt"] * case["Kt"], case["Nc"]), dtype=torch.float64, device="cuda")
    dker = torch.zeros((case["Ng"], case["Nk"], case["Nc"]), dtype=torch.float64, device="cuda")
    slots, choice = x["slots"].long(), x["choice"]
    for g in range(case["Ng"]):
        t, j = torch.nonzero(choice == g, as_tuple=True)
        if t.numel():
            p = slots[t, j]
            d = x["dOut"][p].double()
            din[p] = torch.mm(d, x["Ker"][g].double())
            dker[g] = torch.mm(d.t().contiguous(), x["In"][t].double())
    return [din, dker]


def _exact_adapt(case, x):
    """Each adapter's own weights added up first: Ker + s B A."""
    In, Ker = x["In"].double(), x["Ker"].double()
    out = torch.mm(In, Ker.t().contiguous())
    for a in range(case["Na"]):
        t = torch.nonzero(x["ids"] == a).reshape(-1)
        if t.numel():
            whole = Ker + x["scales"][a].double() * torch.mm(x["B"][a].double(), x["A"][a].double())
            out[t] = torch.mm(In[t], whole.t().contiguous())
    return out


_EXACT = {"route": _exact_route, "combine": _exact_combine, "route_bwd": _exact_route_bwd,
          "group_fwd": _exact_group_fwd, "group_bwd": _exact_group_bwd, "adapt": _exact_adapt}


if __name__ == "__main__":
    for c in listed():
        w = work(c)
        sizes = {k: v for k, v in c.items() if k not in ("name", "op")}
        print(f"{c['name']:15s} {c['op']:10s} {w['flops'] / 1e9:9.3f} GFLOP {w['bytes'] / 1e6:8.2f} MB  {sizes}")
