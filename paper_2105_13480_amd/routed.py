"""Binding of the routed contractions in include/cnn.h: contractions whose Ker
depends on the row.

A router chooses experts for each row (``route``), the rows are multiplied by
their experts' Kers group by group (``group_fwd``), and the results return to
their rows (``combine``); each has its gradient.  ``adapt_fwd`` is a shared
projection with a low-rank adapter for each row.

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
MAX_EXPERTS, MAX_CHOICES = 1024, 16

_torch = None
_types = None  # (operands' dtype, result's dtype) -> cnn_dtype
_here = None
_i32 = _f32 = None


def _load():
    global _torch, _types, _here, _i32, _f32
    import torch
    _types = {(torch.float32, torch.float32): CNN_F32, (torch.bfloat16, torch.float32): CNN_BF16,
              (torch.bfloat16, torch.bfloat16): CNN_BF16_OBF16}
    # the current GPU's index, without the lazy initialisation's check where
    # torch offers that (a call on a small tensor is bound by the host)
    _here = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
    _i32, _f32 = torch.int32, torch.float32
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


def _adapt_own_workspace(In, Ker, A, Out, stream):
    """One for a single call, of the memory of the stream that the call runs on:
    it is free for that stream's later work only."""
    if stream is None:
        return adapt_workspace(In, Ker, A, Out)
    raw = _stream(stream)
    with _torch.cuda.stream(_torch.cuda.ExternalStream(raw) if raw else _torch.cuda.default_stream()):
        return adapt_workspace(In, Ker, A, Out)


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
        ws = _adapt_own_workspace(In, Ker, A, Out, stream)
    st = (cnn._lib or cnn.lib()).cnn_adapt_fwd(
        In.data_ptr(), Ker.data_ptr(), A.data_ptr(), B.data_ptr(), ids.data_ptr(),
        0 if scales is None else scales.data_ptr(), Out.data_ptr(), Nt, Nc, Nk, Na, Nl, dt,
        ws.data_ptr(), ws.numel() * ws.element_size(), _raw(stream))
    if st:
        _check(st)
    return Out
