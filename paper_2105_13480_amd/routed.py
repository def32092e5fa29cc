"""Binding of the routed contractions in include/cnn.h: contractions whose Ker
depends on the row.

A router chooses experts for each row (``route``), the rows are multiplied by
their experts' Kers group by group (``group_fwd``), and the results return to
their rows (``combine``); each has its gradient.  ``adapt_fwd`` is a shared
projection with a low-rank adapter for each row.  ``balance`` counts the router's
choices and gives the losses that keep them even.  ``quantize4`` puts rows into 4
bits with a scale for every 32 values, and ``group_fwd4`` and ``group_bwd_in4``
are the groups' products with such a Ker.

Argument marshalling only, as in ``cnn``: tensors are contiguous torch tensors
on the current GPU, results are the caller's tensors, every call is
asynchronous on the current torch stream unless ``stream`` is given, and
nothing is read back to the host.  A bad shape, type or device raises
ValueError, an error of the library ``cnn.CnnError``.
"""
from __future__ import annotations

import ctypes

from . import cnn
from .cnn import CNN_BF16, CNN_BF16_OBF16, CNN_F32, _check, _stream, i64

OVER = {"all": 0, "chosen": 1}
RULES = {"floor": 0, "up": 1}  # how a block's scale is chosen
MAX_EXPERTS, MAX_CHOICES = 1024, 16

_torch = None
_types = None  # (operands' dtype, result's dtype) -> cnn_dtype
_here = None
_i32 = _f32 = _u8 = None


def _load():
    global _torch, _types, _here, _i32, _f32, _u8
    import torch
    _types = {(torch.float32, torch.float32): CNN_F32, (torch.bfloat16, torch.float32): CNN_BF16,
              (torch.bfloat16, torch.bfloat16): CNN_BF16_OBF16}
    # the current GPU's index, without the lazy initialisation's check where
    # torch offers that (a call on a small tensor is bound by the host)
    _here = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
    _i32, _f32, _u8 = torch.int32, torch.float32, torch.uint8
    _torch = torch
    return torch


def _refuse(**tensors):
    """Name what is wrong with the tensors of a call (None is left out)."""
    here = _torch.cuda.current_device()
    for name, t in tensors.items():
        if t is None:
            continue
        if not t.is_cuda or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous GPU tensor")
        if t.get_device() != here:
            raise ValueError(f"{name} is on GPU {t.get_device()}, the current one is {here}")


def _shape(name, t, *shape):
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {shape}, not {tuple(t.shape)}")


def _dims(name, t, n):
    shape = t.shape
    if len(shape) != n:
        raise ValueError(f"{name} must be {n}-d")
    return shape


def _of(dtype, **tensors):
    for name, t in tensors.items():
        if t is not None and t.dtype is not dtype:
            raise ValueError(f"{name} must be {dtype}")


def _dtype(result, *operands):
    """cnn_dtype of operands of one type and their result."""
    ti = operands[0].dtype
    dt = _types.get((ti, result.dtype))
    if dt is None:
        raise ValueError("operands must all be float32 or all bfloat16, results float32 or, of "
                         "bfloat16 operands, bfloat16")
    for t in operands:
        if t.dtype is not ti:
            raise ValueError("operands must all be float32 or all bfloat16")
    return dt


def _order(offsets, rows, Np, Ng):
    _shape("offsets", offsets, Ng + 1)
    _of(_i32, offsets=offsets, rows=rows)
    if rows is not None:
        _shape("rows", rows, Np)


def _enter():
    """The current GPU's index, with torch loaded."""
    if _torch is None:
        _load()
    return _here()


def _raw(stream):
    """A stream argument as the library takes it; None: the current stream."""
    if stream is None and cnn._raw_stream is not None:
        return cnn._raw_stream(_here())
    return _stream(stream)


class Routing:
    """What ``route`` fills for Nt rows, Ng experts and Kt choices of a row,
    with its workspace: kept and reused by a program as long as these sizes
    hold.

    ``choice`` [Nt, Kt] int32 (-1: none), ``gates`` [Nt, Kt] float32,
    ``offsets`` [Ng + 1], ``rows`` [Nt Kt] and ``slots`` [Nt, Kt] int32: the
    (row, choice) pairs in the order of their experts.
    """

    def __init__(self, Nt: int, Ng: int, Kt: int, device=None):
        _enter()
        torch = _torch
        n = i64()
        _check(cnn.lib().cnn_route_ws(Nt, Ng, Kt, ctypes.byref(n)))
        device = torch.device("cuda", torch.cuda.current_device()) if device is None else device
        self.Nt, self.Ng, self.Kt = Nt, Ng, Kt
        self.choice = torch.empty((Nt, Kt), dtype=torch.int32, device=device)
        self.gates = torch.empty((Nt, Kt), dtype=torch.float32, device=device)
        self.offsets = torch.empty(Ng + 1, dtype=torch.int32, device=device)
        self.rows = torch.empty(Nt * Kt, dtype=torch.int32, device=device)
        self.slots = torch.empty((Nt, Kt), dtype=torch.int32, device=device)
        self.ws = torch.empty(n.value, dtype=torch.uint8, device=device) if n.value else None
        self.shape, self.ws_bytes = (Nt, Ng), n.value


def route(Logits, routing: Routing, over: str = "chosen", stream=None) -> Routing:
    """Choose the Kt experts of each row of Logits [Nt, Ng] (float32 or
    bfloat16) and order the pairs; fills and returns ``routing``.  ``over``:
    the weights are a softmax over "all" allowed experts or over the "chosen"
    ones.  Experts with logit -inf or NaN are never chosen."""
    r = routing
    here = _enter()
    choice = r.choice
    if not (Logits.get_device() == here == choice.get_device() and Logits.is_contiguous()
            and Logits.shape == r.shape and over in OVER):
        _refuse(Logits=Logits, routing=choice)
        _shape("Logits", Logits, r.Nt, r.Ng)
        raise ValueError(f"over must be one of {sorted(OVER)}")
    dt = _types.get((Logits.dtype, Logits.dtype))
    if dt is None:
        raise ValueError("Logits must be float32 or bfloat16")
    st = (cnn._lib or cnn.lib()).cnn_route(
        Logits.data_ptr(), choice.data_ptr(), r.gates.data_ptr(), r.offsets.data_ptr(),
        r.rows.data_ptr(), r.slots.data_ptr(), r.Nt, r.Ng, r.Kt, dt, OVER[over],
        0 if r.ws is None else r.ws.data_ptr(), r.ws_bytes, _raw(stream))
    if st:
        _check(st)
    return r


def route_bwd(Logits, choice, gates, dGates, dLogits, over: str = "chosen", stream=None):
    """dLogits from dGates, for the choice and gates that ``route`` gave with
    the same ``over``."""
    here = _enter()
    Nt, Ng = _dims("Logits", Logits, 2)
    pairs = choice.shape
    if not (Logits.get_device() == here == choice.get_device() == gates.get_device() ==
            dGates.get_device() == dLogits.get_device() and Logits.is_contiguous()
            and choice.is_contiguous() and gates.is_contiguous() and dGates.is_contiguous()
            and dLogits.is_contiguous() and len(pairs) == 2 and pairs[0] == Nt
            and gates.shape == pairs == dGates.shape and dLogits.shape == Logits.shape
            and choice.dtype is _i32 and gates.dtype is _f32 is dGates.dtype and over in OVER):
        _refuse(Logits=Logits, choice=choice, gates=gates, dGates=dGates, dLogits=dLogits)
        Kt = _dims("choice", choice, 2)[1]
        _shape("choice", choice, Nt, Kt)
        _shape("gates", gates, Nt, Kt)
        _shape("dGates", dGates, Nt, Kt)
        _shape("dLogits", dLogits, Nt, Ng)
        _of(_i32, choice=choice)
        _of(_f32, gates=gates, dGates=dGates)
        raise ValueError(f"over must be one of {sorted(OVER)}")
    dt = _dtype(dLogits, Logits)
    st = (cnn._lib or cnn.lib()).cnn_route_bwd(
        Logits.data_ptr(), choice.data_ptr(), gates.data_ptr(), dGates.data_ptr(),
        dLogits.data_ptr(), Nt, Ng, pairs[1], dt, OVER[over], _raw(stream))
    if st:
        _check(st)
    return dLogits


def combine(In, Out, slots, gates=None, stream=None):
    """Out[t] = sum_j gates[t, j] In[slots[t, j]] (gates None: ones; slot -1
    adds nothing).  Without gates it sums dIn of ``group_bwd_in`` over a row's
    places: the gradient of the gather."""
    here = _enter()
    Np, Nk = _dims("In", In, 2)
    Nt, Kt = _dims("slots", slots, 2)
    if not (In.get_device() == here == Out.get_device() == slots.get_device()
            and In.is_contiguous() and Out.is_contiguous() and slots.is_contiguous()
            and Out.shape == (Nt, Nk) and slots.dtype is _i32
            and (gates is None or (gates.get_device() == here and gates.is_contiguous()
                                   and gates.shape == slots.shape and gates.dtype is _f32))):
        _refuse(In=In, Out=Out, slots=slots, gates=gates)
        _shape("Out", Out, Nt, Nk)
        _of(_i32, slots=slots)
        _shape("gates", gates, Nt, Kt)
        _of(_f32, gates=gates)
    dt = _dtype(Out, In)
    st = (cnn._lib or cnn.lib()).cnn_combine(
        In.data_ptr(), slots.data_ptr(), 0 if gates is None else gates.data_ptr(), Out.data_ptr(),
        Nt, Kt, Np, Nk, dt, _raw(stream))
    if st:
        _check(st)
    return Out


def combine_bwd(dOut, In, dIn, dGates, slots, rows, gates=None, stream=None):
    """dIn[p] = gate dOut[t] and dGates[t, j] = dOut[t] . In[p] for p =
    slots[t, j], t = rows[p]; dIn is zero at the places without a pair (rows[p]
    < 0), dGates for the choices without a place.  dGates None: not wanted."""
    here = _enter()
    Np, Nk = _dims("In", In, 2)
    Nt, Kt = _dims("slots", slots, 2)
    if not (dOut.get_device() == here == In.get_device() == dIn.get_device() == slots.get_device() ==
            rows.get_device() and dOut.is_contiguous() and In.is_contiguous()
            and dIn.is_contiguous() and slots.is_contiguous() and rows.is_contiguous()
            and dOut.shape == (Nt, Nk) and dIn.shape == In.shape and rows.shape == (Np,)
            and slots.dtype is _i32 is rows.dtype
            and (gates is None or (gates.get_device() == here and gates.is_contiguous()
                                   and gates.shape == slots.shape and gates.dtype is _f32))
            and (dGates is None or (dGates.get_device() == here and dGates.is_contiguous()
                                    and dGates.shape == slots.shape and dGates.dtype is _f32))):
        _refuse(dOut=dOut, In=In, dIn=dIn, dGates=dGates, slots=slots, rows=rows, gates=gates)
        _shape("dOut", dOut, Nt, Nk)
        _shape("dIn", dIn, Np, Nk)
        _shape("rows", rows, Np)
        _of(_i32, slots=slots, rows=rows)
        for name, t in (("gates", gates), ("dGates", dGates)):
            if t is not None:
                _shape(name, t, Nt, Kt)
                _of(_f32, **{name: t})
    dt = _dtype(dIn, dOut, In)
    st = (cnn._lib or cnn.lib()).cnn_combine_bwd(
        dOut.data_ptr(), In.data_ptr(), slots.data_ptr(), rows.data_ptr(),
        0 if gates is None else gates.data_ptr(), dIn.data_ptr(),
        0 if dGates is None else dGates.data_ptr(), Nt, Kt, Np, Nk, dt, _raw(stream))
    if st:
        _check(st)
    return dIn, dGates


def group_fwd(In, Ker, Out, offsets, rows=None, stream=None):
    """Out[p] = In[rows[p]] Ker[g]^T for the places p of group g
    ([offsets[g], offsets[g+1])): In [Nt, Nc], Ker [Ng, Nk, Nc], Out [Np, Nk].
    rows None: In is in grouped order.  Places past offsets[Ng] get zeros."""
    here = _enter()
    Nt, Nc = _dims("In", In, 2)
    Ng, Nk, C = _dims("Ker", Ker, 3)
    Np, K = _dims("Out", Out, 2)
    if not (In.get_device() == here == Ker.get_device() == Out.get_device() == offsets.get_device()
            and In.is_contiguous() and Ker.is_contiguous() and Out.is_contiguous()
            and offsets.is_contiguous() and C == Nc and K == Nk and offsets.shape == (Ng + 1,)
            and offsets.dtype is _i32
            and (Np == Nt if rows is None else
                 rows.get_device() == here and rows.is_contiguous() and rows.dtype is _i32
                 and rows.shape == (Np,))):
        _refuse(In=In, Ker=Ker, Out=Out, offsets=offsets, rows=rows)
        _shape("Ker", Ker, Ng, Nk, Nc)
        _shape("Out", Out, Nt if rows is None else Np, Nk)
        _order(offsets, rows, Np, Ng)
    dt = _dtype(Out, In, Ker)
    st = (cnn._lib or cnn.lib()).cnn_group_fwd(
        In.data_ptr(), Ker.data_ptr(), Out.data_ptr(), offsets.data_ptr(),
        0 if rows is None else rows.data_ptr(), Nt, Np, Ng, Nc, Nk, dt, _raw(stream))
    if st:
        _check(st)
    return Out


def group_bwd_in(dOut, Ker, dIn, offsets, stream=None):
    """dIn[p] = dOut[p] Ker[g], in grouped order: dOut [Np, Nk], Ker
    [Ng, Nk, Nc], dIn [Np, Nc].  ``combine`` without gates adds up a gathered
    row's places."""
    here = _enter()
    Np, Nk = _dims("dOut", dOut, 2)
    Ng, K, Nc = _dims("Ker", Ker, 3)
    if not (dOut.get_device() == here == Ker.get_device() == dIn.get_device() == offsets.get_device()
            and dOut.is_contiguous() and Ker.is_contiguous() and dIn.is_contiguous()
            and offsets.is_contiguous() and K == Nk and dIn.shape == (Np, Nc)
            and offsets.shape == (Ng + 1,) and offsets.dtype is _i32):
        _refuse(dOut=dOut, Ker=Ker, dIn=dIn, offsets=offsets)
        _shape("Ker", Ker, Ng, Nk, Nc)
        _shape("dIn", dIn, Np, Nc)
        _order(offsets, None, Np, Ng)
    dt = _dtype(dIn, dOut, Ker)
    st = (cnn._lib or cnn.lib()).cnn_group_bwd_in(dOut.data_ptr(), Ker.data_ptr(), dIn.data_ptr(),
                                                  offsets.data_ptr(), Np, Ng, Nc, Nk, dt,
                                                  _raw(stream))
    if st:
        _check(st)
    return dIn


def group_bwd_ker(dOut, In, dKer, offsets, rows=None, stream=None):
    """dKer[g] = sum over group g's places p of dOut[p]^T In[rows[p]]: dOut
    [Np, Nk], In [Nt, Nc], dKer [Ng, Nk, Nc]; zeros for an empty group."""
    here = _enter()
    Np, Nk = _dims("dOut", dOut, 2)
    Nt, Nc = _dims("In", In, 2)
    Ng, K, C = _dims("dKer", dKer, 3)
    if not (dOut.get_device() == here == In.get_device() == dKer.get_device() == offsets.get_device()
            and dOut.is_contiguous() and In.is_contiguous() and dKer.is_contiguous()
            and offsets.is_contiguous() and K == Nk and C == Nc and offsets.shape == (Ng + 1,)
            and offsets.dtype is _i32
            and (Np == Nt if rows is None else
                 rows.get_device() == here and rows.is_contiguous() and rows.dtype is _i32
                 and rows.shape == (Np,))):
        _refuse(dOut=dOut, In=In, dKer=dKer, offsets=offsets, rows=rows)
        _shape("dKer", dKer, Ng, Nk, Nc)
        _shape("In", In, Np if rows is None else Nt, Nc)
        _order(offsets, rows, Np, Ng)
    dt = _dtype(dKer, dOut, In)
    st = (cnn._lib or cnn.lib()).cnn_group_bwd_ker(
        dOut.data_ptr(), In.data_ptr(), dKer.data_ptr(), offsets.data_ptr(),
        0 if rows is None else rows.data_ptr(), Nt, Np, Ng, Nc, Nk, dt, _raw(stream))
    if st:
        _check(st)
    return dKer


def _adapt_dims(In, Ker, A, Out):
    Nt, Nc = _dims("In", In, 2)
    Nk = _dims("Ker", Ker, 2)[0]
    Na, Nl, _ = _dims("A", A, 3)
    _shape("Ker", Ker, Nk, Nc)
    _shape("A", A, Na, Nl, Nc)
    _shape("Out", Out, Nt, Nk)
    return Nt, Nc, Nk, Na, Nl


def adapt_workspace(In, Ker, A, Out):
    """A workspace for ``adapt_fwd`` on tensors of these shapes."""
    _enter()
    n = i64()
    _check(cnn.lib().cnn_adapt_ws(*_adapt_dims(In, Ker, A, Out), ctypes.byref(n)))
    return _torch.empty(n.value, dtype=_torch.uint8, device=In.device)


def _own_workspace(make, stream):
    """One for a single call, of the memory of the stream that the call runs on:
    it is free for that stream's later work only."""
    if stream is None:
        return make()
    raw = _stream(stream)
    with _torch.cuda.stream(_torch.cuda.ExternalStream(raw) if raw else _torch.cuda.default_stream()):
        return make()


def adapt_fwd(In, Ker, A, B, ids, Out, scales=None, ws=None, stream=None):
    """Out[t] = In[t] Ker^T + scales[a] (In[t] A[a]^T) B[a]^T with a = ids[t]
    (outside [0, Na): no adapter): In [Nt, Nc], Ker [Nk, Nc], A [Na, Nl, Nc],
    B [Na, Nk, Nl], scales [Na] float32 (None: ones).  ws: the tensor that
    ``adapt_workspace`` gives, kept by the caller (None: one of its own for
    this call)."""
    here = _enter()
    Nt, Nc, Nk, Na, Nl = _adapt_dims(In, Ker, A, Out)
    if not (In.get_device() == here == Ker.get_device() == A.get_device() == B.get_device() ==
            ids.get_device() == Out.get_device() and In.is_contiguous() and Ker.is_contiguous()
            and A.is_contiguous() and B.is_contiguous() and ids.is_contiguous()
            and Out.is_contiguous() and B.shape == (Na, Nk, Nl) and ids.shape == (Nt,)
            and ids.dtype is _i32
            and (scales is None or (scales.get_device() == here and scales.is_contiguous()
                                    and scales.shape == (Na,) and scales.dtype is _f32))
            and (ws is None or (ws.get_device() == here and ws.is_contiguous()))):
        _refuse(In=In, Ker=Ker, A=A, B=B, ids=ids, Out=Out, scales=scales, ws=ws)
        _shape("B", B, Na, Nk, Nl)
        _shape("ids", ids, Nt)
        _of(_i32, ids=ids)
        _shape("scales", scales, Na)
        _of(_f32, scales=scales)
    dt = _dtype(Out, In, Ker, A, B)
    if ws is None:
        ws = _own_workspace(lambda: adapt_workspace(In, Ker, A, Out), stream)
    st = (cnn._lib or cnn.lib()).cnn_adapt_fwd(
        In.data_ptr(), Ker.data_ptr(), A.data_ptr(), B.data_ptr(), ids.data_ptr(),
        0 if scales is None else scales.data_ptr(), Out.data_ptr(), Nt, Nc, Nk, Na, Nl, dt,
        ws.data_ptr(), ws.numel() * ws.element_size(), _raw(stream))
    if st:
        _check(st)
    return Out


def balance_workspace(Nt: int, Ng: int, Ns: int = 1, device=None):
    """A workspace for ``balance`` of Nt rows, Ng experts and Ns sequences (None
    where it needs none)."""
    _enter()
    n = i64()
    _check(cnn.lib().cnn_balance_ws(Nt, Ng, Ns, ctypes.byref(n)))
    device = _torch.device("cuda", _torch.cuda.current_device()) if device is None else device
    return _torch.empty(n.value, dtype=_u8, device=device) if n.value else None


def _balance_check(here, Logits, choice, counts, tokens, bounds, name, pair):
    """Of balance and balance_bwd (pair: the two losses or their gradients): Nt, Ng,
    Kt, Ns."""
    shape, pairs, table = Logits.shape, choice.shape, counts.shape
    if (Logits.get_device() == here == choice.get_device() == counts.get_device() == tokens.get_device() ==
            pair.get_device() and len(shape) == 2 == len(pairs) and len(table) == 2 and pairs[0] == shape[0]
            and table[1] == shape[1] and tokens.shape == (table[0],) and pair.shape == (2,)
            and choice.dtype is _i32 is counts.dtype and tokens.dtype is _i32 and pair.dtype is _f32
            and Logits.is_contiguous() and choice.is_contiguous() and counts.is_contiguous()
            and tokens.is_contiguous() and pair.is_contiguous()
            and (bounds is None or (bounds.get_device() == here and bounds.is_contiguous()
                                    and bounds.shape == (table[0] + 1,) and bounds.dtype is _i32))):
        return shape[0], shape[1], pairs[1], table[0]
    Nt, Ng = _dims("Logits", Logits, 2)
    Kt = _dims("choice", choice, 2)[1]
    Ns = _dims("counts", counts, 2)[0]
    _refuse(Logits=Logits, choice=choice, counts=counts, tokens=tokens, bounds=bounds, **{name: pair})
    _shape("choice", choice, Nt, Kt)
    _shape("counts", counts, Ns, Ng)
    _shape("tokens", tokens, Ns)
    _shape(name, pair, 2)
    _of(_i32, choice=choice, counts=counts, tokens=tokens, bounds=bounds)
    _of(_f32, **{name: pair})
    _shape("bounds", bounds, Ns + 1)


def balance(Logits, choice, counts, tokens, loss, bounds=None, ws=None, stream=None):
    """The choices of each expert and the losses that keep them even: for Logits
    [Nt, Ng], the choice [Nt, Kt] that ``route`` made of them and sequences of the
    rows [bounds[s], bounds[s + 1]) (bounds [Ns + 1] int32; None: one of all
    rows), counts [Ns, Ng] and tokens [Ns] int32 (rows with a choice) and loss [2]
    float32: the balance loss, 1 where the choices are even, and the mean square
    of the rows' log-sum-exp.  ws: the tensor that ``balance_workspace`` gives,
    kept by the caller (None: one of its own for this call, if it needs any)."""
    here = _enter()
    Nt, Ng, Kt, Ns = _balance_check(here, Logits, choice, counts, tokens, bounds, "loss", loss)
    dt = _types.get((Logits.dtype, Logits.dtype))
    if dt is None:
        raise ValueError("Logits must be float32 or bfloat16")
    if ws is None:
        ws = _own_workspace(lambda: balance_workspace(Nt, Ng, Ns), stream)
    elif ws.get_device() != here or not ws.is_contiguous():
        _refuse(ws=ws)
    st = (cnn._lib or cnn.lib()).cnn_balance(
        Logits.data_ptr(), choice.data_ptr(), 0 if bounds is None else bounds.data_ptr(),
        counts.data_ptr(), tokens.data_ptr(), loss.data_ptr(), Nt, Ng, Kt, Ns, dt,
        0 if ws is None else ws.data_ptr(), 0 if ws is None else ws.numel() * ws.element_size(),
        _raw(stream))
    if st:
        _check(st)
    return loss


def balance_bwd(Logits, choice, counts, tokens, dLoss, dLogits, bounds=None, add=False, stream=None):
    """dLogits of dLoss[0] loss[0] + dLoss[1] loss[1], dLoss [2] float32 on the
    GPU, for the counts and tokens that ``balance`` gave; add: on top of what
    dLogits holds (what ``route_bwd`` wrote)."""
    here = _enter()
    Nt, Ng, Kt, Ns = _balance_check(here, Logits, choice, counts, tokens, bounds, "dLoss", dLoss)
    if not (dLogits.get_device() == here and dLogits.is_contiguous() and dLogits.shape == Logits.shape):
        _refuse(dLogits=dLogits)
        _shape("dLogits", dLogits, Nt, Ng)
    dt = _dtype(dLogits, Logits)
    st = (cnn._lib or cnn.lib()).cnn_balance_bwd(
        Logits.data_ptr(), choice.data_ptr(), 0 if bounds is None else bounds.data_ptr(),
        counts.data_ptr(), tokens.data_ptr(), dLoss.data_ptr(), dLogits.data_ptr(), Nt, Ng, Kt, Ns,
        dt, int(bool(add)), _raw(stream))
    if st:
        _check(st)
    return dLogits


def blocks4(Nc: int) -> int:
    """Blocks of a row of Nc values in 4 bits: 16 bytes of codes and one of scale each."""
    return (Nc + 31) // 32


def _four(here, name, codes, scales, lead, Nb):
    """Refuses what is no tensor in 4 bits of sizes `lead` and Nb blocks on this GPU."""
    if not (codes.get_device() == here == scales.get_device() and codes.dtype is _u8 is scales.dtype
            and codes.shape == (*lead, 16 * Nb) and scales.shape == (*lead, Nb)
            and codes.is_contiguous() and scales.is_contiguous()):
        _refuse(**{name: codes, name + "Scales": scales})
        _of(_u8, **{name: codes, name + "Scales": scales})
        _shape(name, codes, *lead, 16 * Nb)
        _shape(name + "Scales", scales, *lead, Nb)


def _rows_of(name, t):
    """Leading sizes, their product and columns of a tensor of values."""
    shape = t.shape
    if not shape:
        raise ValueError(f"{name} must be at least 1-d")
    if len(shape) == 2:
        return shape[:1], shape[0], shape[1]
    lead, rows = shape[:-1], 1
    for n in lead:
        rows *= n
    return lead, rows, shape[-1]


def quantize4(In, Codes, Scales, rule: str = "floor", stream=None):
    """In [.., Nc] (float32 or bfloat16) in 4 bits: Codes [.., 16 blocks4(Nc)] and
    Scales [.., blocks4(Nc)] uint8.  rule: a block's scale is a power of two,
    "floor" of a quarter of its largest magnitude (up to a fourth of it is cut
    off) or "up", so that nothing is.  A block with an infinity or NaN becomes
    NaN.  Returns Codes and Scales."""
    here = _enter()
    lead, Nt, Nc = _rows_of("In", In)
    if not (In.get_device() == here and In.is_contiguous() and rule in RULES):
        _refuse(In=In)
        raise ValueError(f"rule must be one of {sorted(RULES)}")
    _four(here, "Codes", Codes, Scales, lead, (Nc + 31) // 32)
    dt = _types.get((In.dtype, In.dtype))
    if dt is None:
        raise ValueError("In must be float32 or bfloat16")
    st = (cnn._lib or cnn.lib()).cnn_quantize4(In.data_ptr(), Codes.data_ptr(), Scales.data_ptr(), Nt,
                                               Nc, dt, RULES[rule], _raw(stream))
    if st:
        _check(st)
    return Codes, Scales


def dequantize4(Codes, Scales, Out, stream=None):
    """The values of a tensor in 4 bits, Out [.., Nc] float32 or bfloat16
    (exact in both; from 2^128 on infinite)."""
    here = _enter()
    lead, Nt, Nc = _rows_of("Out", Out)
    if not (Out.get_device() == here and Out.is_contiguous()):
        _refuse(Out=Out)
    _four(here, "Codes", Codes, Scales, lead, (Nc + 31) // 32)
    dt = _types.get((Out.dtype, Out.dtype))
    if dt is None:
        raise ValueError("Out must be float32 or bfloat16")
    st = (cnn._lib or cnn.lib()).cnn_dequantize4(Codes.data_ptr(), Scales.data_ptr(), Out.data_ptr(),
                                                 Nt, Nc, dt, _raw(stream))
    if st:
        _check(st)
    return Out


def _result4(name, t):
    if t.dtype is _torch.bfloat16:
        return CNN_BF16_OBF16
    if t.dtype is _f32:
        return CNN_BF16
    raise ValueError(f"{name} must be float32 or bfloat16")


def group_fwd4(In, Ker, KerScales, Out, offsets, rows=None, InScales=None, stream=None):
    """``group_fwd`` with Ker in 4 bits: Ker [Ng, Nk, 16 Nb], KerScales [Ng, Nk, Nb]
    as ``quantize4`` makes them of [Ng, Nk, Nc].  In [Nt, Nc] bfloat16, or in 4
    bits itself: In [Nt, 16 Nb] with InScales [Nt, Nb].  Out float32 or bfloat16."""
    here = _enter()
    Ng, Nk, _ = _dims("Ker", Ker, 3)
    Np, K = _dims("Out", Out, 2)
    Nt, Nc = _dims("In", In, 2)
    if InScales is not None:
        Nc = 32 * _dims("InScales", InScales, 2)[1]
        _four(here, "In", In, InScales, (Nt,), Nc // 32)
    elif In.dtype is not _torch.bfloat16:
        raise ValueError("In must be bfloat16, or uint8 with InScales")
    _four(here, "Ker", Ker, KerScales, (Ng, Nk), (Nc + 31) // 32)
    if not (In.get_device() == here == Out.get_device() == offsets.get_device()
            and In.is_contiguous() and Out.is_contiguous() and offsets.is_contiguous() and K == Nk
            and offsets.shape == (Ng + 1,) and offsets.dtype is _i32
            and (Np == Nt if rows is None else
                 rows.get_device() == here and rows.is_contiguous() and rows.dtype is _i32
                 and rows.shape == (Np,))):
        _refuse(In=In, Out=Out, offsets=offsets, rows=rows)
        _shape("Out", Out, Nt if rows is None else Np, Nk)
        _order(offsets, rows, Np, Ng)
    st = (cnn._lib or cnn.lib()).cnn_group_fwd4(
        In.data_ptr(), 0 if InScales is None else InScales.data_ptr(), Ker.data_ptr(),
        KerScales.data_ptr(), Out.data_ptr(), offsets.data_ptr(), 0 if rows is None else rows.data_ptr(),
        Nt, Np, Ng, Nc, Nk, _result4("Out", Out), _raw(stream))
    if st:
        _check(st)
    return Out


def group_bwd_in4(dOut, Ker, KerScales, dIn, offsets, stream=None):
    """``group_bwd_in`` with Ker in 4 bits (along c, as ``group_fwd4`` takes it):
    dOut [Np, Nk] bfloat16, dIn [Np, Nc] float32 or bfloat16."""
    here = _enter()
    Np, Nk = _dims("dOut", dOut, 2)
    Ng, _, _ = _dims("Ker", Ker, 3)
    Nc = _dims("dIn", dIn, 2)[1]
    _four(here, "Ker", Ker, KerScales, (Ng, Nk), (Nc + 31) // 32)
    if not (dOut.get_device() == here == dIn.get_device() == offsets.get_device()
            and dOut.is_contiguous() and dIn.is_contiguous() and offsets.is_contiguous()
            and dIn.shape == (Np, Nc) and offsets.shape == (Ng + 1,) and offsets.dtype is _i32):
        _refuse(dOut=dOut, dIn=dIn, offsets=offsets)
        _shape("dIn", dIn, Np, Nc)
        _order(offsets, None, Np, Ng)
    if dOut.dtype is not _torch.bfloat16:
        raise ValueError("dOut must be bfloat16")
    st = (cnn._lib or cnn.lib()).cnn_group_bwd_in4(
        dOut.data_ptr(), Ker.data_ptr(), KerScales.data_ptr(), dIn.data_ptr(), offsets.data_ptr(), Np,
        Ng, Nc, Nk, _result4("dIn", dIn), _raw(stream))
    if st:
        _check(st)
    return dIn
