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


def _load():
    global _torch, _types, _here
    import torch
    _types = {(torch.float32, torch.float32): CNN_F32, (torch.bfloat16, torch.float32): CNN_BF16,
              (torch.bfloat16, torch.bfloat16): CNN_BF16_OBF16}
    # the current GPU's index, without the lazy initialisation's check where
    # torch offers that (a call on a small tensor is bound by the host)
    _here = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
    _torch = torch
    return torch


def _lib():
    return cnn._lib or cnn.lib()


def _same(here, *tensors):
    """Whether all are contiguous tensors on GPU `here`."""
    for t in tensors:
        if t.get_device() != here or not t.is_contiguous():
            return False
    return True


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


def _ptr(t):
    return 0 if t is None else t.data_ptr()


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
        _check(_lib().cnn_route_ws(Nt, Ng, Kt, ctypes.byref(n)))
        device = torch.device("cuda", torch.cuda.current_device()) if device is None else device
        self.Nt, self.Ng, self.Kt = Nt, Ng, Kt
        self.choice = torch.empty((Nt, Kt), dtype=torch.int32, device=device)
        self.gates = torch.empty((Nt, Kt), dtype=torch.float32, device=device)
        self.offsets = torch.empty(Ng + 1, dtype=torch.int32, device=device)
        self.rows = torch.empty(Nt * Kt, dtype=torch.int32, device=device)
        self.slots = torch.empty((Nt, Kt), dtype=torch.int32, device=device)
        self.ws = torch.empty(n.value, dtype=torch.uint8, device=device) if n.value else None


def route(Logits, routing: Routing, over: str = "chosen", stream=None) -> Routing:
    """Choose the Kt experts of each row of Logits [Nt, Ng] (float32 or
    bfloat16) and order the pairs; fills and returns ``routing``.  ``over``:
    the weights are a softmax over "all" allowed experts or over the "chosen"
    ones.  Experts with logit -inf or NaN are never chosen."""
    r = routing
    if not _same(_enter(), Logits, r.choice):
        _refuse(Logits=Logits, routing=r.choice)
    _shape("Logits", Logits, r.Nt, r.Ng)
    if over not in OVER:
        raise ValueError(f"over must be one of {sorted(OVER)}")
    dt = _dtype(Logits, Logits)
    ws = r.ws
    st = _lib().cnn_route(Logits.data_ptr(), r.choice.data_ptr(), r.gates.data_ptr(),
                          r.offsets.data_ptr(), r.rows.data_ptr(), r.slots.data_ptr(), r.Nt, r.Ng,
                          r.Kt, dt, OVER[over], _ptr(ws), 0 if ws is None else ws.numel(),
                          _raw(stream))
    if st:
        _check(st)
    return r


def route_bwd(Logits, choice, gates, dGates, dLogits, over: str = "chosen", stream=None):
    """dLogits from dGates, for the choice and gates that ``route`` gave with
    the same ``over``."""
    if not _same(_enter(), Logits, choice, gates, dGates, dLogits):
        _refuse(Logits=Logits, choice=choice, gates=gates, dGates=dGates, dLogits=dLogits)
    Nt, Ng = _dims("Logits", Logits, 2)
    Kt = _dims("choice", choice, 2)[1]
    _shape("choice", choice, Nt, Kt)
    _shape("gates", gates, Nt, Kt)
    _shape("dGates", dGates, Nt, Kt)
    _shape("dLogits", dLogits, Nt, Ng)
    _of(_torch.int32, choice=choice)
    _of(_torch.float32, gates=gates, dGates=dGates)
    if over not in OVER:
        raise ValueError(f"over must be one of {sorted(OVER)}")
    dt = _dtype(dLogits, Logits)
    st = _lib().cnn_route_bwd(Logits.data_ptr(), choice.data_ptr(), gates.data_ptr(),
                              dGates.data_ptr(), dLogits.data_ptr(), Nt, Ng, Kt, dt, OVER[over],
                              _raw(stream))
    if st:
        _check(st)
    return dLogits


def combine(In, Out, slots, gates=None, stream=None):
    """Out[t] = sum_j gates[t, j] In[slots[t, j]] (gates None: ones; slot -1
    adds nothing).  Without gates it sums dIn of ``group_bwd_in`` over a row's
    places: the gradient of the gather."""
    if not _same(_enter(), In, Out, slots, slots if gates is None else gates):
        _refuse(In=In, Out=Out, slots=slots, gates=gates)
    Np, Nk = _dims("In", In, 2)
    Nt, Kt = _dims("slots", slots, 2)
    _shape("Out", Out, Nt, Nk)
    _of(_torch.int32, slots=slots)
    if gates is not None:
        _shape("gates", gates, Nt, Kt)
        _of(_torch.float32, gates=gates)
    dt = _dtype(Out, In)
    st = _lib().cnn_combine(In.data_ptr(), slots.data_ptr(), _ptr(gates), Out.data_ptr(), Nt, Kt,
                            Np, Nk, dt, _raw(stream))
    if st:
        _check(st)
    return Out


def combine_bwd(dOut, In, dIn, dGates, slots, rows, gates=None, stream=None):
    """dIn[p] = gate dOut[t] and dGates[t, j] = dOut[t] . In[p] for p =
    slots[t, j]; dIn is zero at the places without a pair (rows[p] < 0).
    dGates None: not wanted."""
    if not _same(_enter(), dOut, In, dIn, slots, rows, slots if gates is None else gates,
                 slots if dGates is None else dGates):
        _refuse(dOut=dOut, In=In, dIn=dIn, dGates=dGates, slots=slots, rows=rows, gates=gates)
    Np, Nk = _dims("In", In, 2)
    Nt, Kt = _dims("slots", slots, 2)
    _shape("dOut", dOut, Nt, Nk)
    _shape("dIn", dIn, Np, Nk)
    _shape("rows", rows, Np)
    _of(_torch.int32, slots=slots, rows=rows)
    for name, t in (("gates", gates), ("dGates", dGates)):
        if t is not None:
            _shape(name, t, Nt, Kt)
            _of(_torch.float32, **{name: t})
    dt = _dtype(dIn, dOut, In)
    st = _lib().cnn_combine_bwd(dOut.data_ptr(), In.data_ptr(), slots.data_ptr(), rows.data_ptr(),
                                _ptr(gates), dIn.data_ptr(), _ptr(dGates), Nt, Kt, Np, Nk, dt,
                                _raw(stream))
    if st:
        _check(st)
    return dIn, dGates


def _group(offsets, rows, Np, Ng):
    _shape("offsets", offsets, Ng + 1)
    _of(_torch.int32, offsets=offsets, rows=rows)
    if rows is not None:
        _shape("rows", rows, Np)


def group_fwd(In, Ker, Out, offsets, rows=None, stream=None):
    """Out[p] = In[rows[p]] Ker[g]^T for the places p of group g
    ([offsets[g], offsets[g+1])): In [Nt, Nc], Ker [Ng, Nk, Nc], Out [Np, Nk].
    rows None: In is in grouped order.  Places past offsets[Ng] get zeros."""
    if not _same(_enter(), In, Ker, Out, offsets, offsets if rows is None else rows):
        _refuse(In=In, Ker=Ker, Out=Out, offsets=offsets, rows=rows)
    Nt, Nc = _dims("In", In, 2)
    Ng, Nk, _ = _dims("Ker", Ker, 3)
    Np = _dims("Out", Out, 2)[0]
    _shape("Ker", Ker, Ng, Nk, Nc)
    _shape("Out", Out, Np if rows is not None else Nt, Nk)
    _group(offsets, rows, Np, Ng)
    dt = _dtype(Out, In, Ker)
    st = _lib().cnn_group_fwd(In.data_ptr(), Ker.data_ptr(), Out.data_ptr(), offsets.data_ptr(),
                              _ptr(rows), Nt, Np, Ng, Nc, Nk, dt, _raw(stream))
    if st:
        _check(st)
    return Out


def group_bwd_in(dOut, Ker, dIn, offsets, stream=None):
    """dIn[p] = dOut[p] Ker[g], in grouped order: dOut [Np, Nk], Ker
    [Ng, Nk, Nc], dIn [Np, Nc].  ``combine`` without gates adds up a gathered
    row's places."""
    if not _same(_enter(), dOut, Ker, dIn, offsets):
        _refuse(dOut=dOut, Ker=Ker, dIn=dIn, offsets=offsets)
    Np, Nk = _dims("dOut", dOut, 2)
    Ng, _, Nc = _dims("Ker", Ker, 3)
    _shape("Ker", Ker, Ng, Nk, Nc)
    _shape("dIn", dIn, Np, Nc)
    _group(offsets, None, Np, Ng)
    dt = _dtype(dIn, dOut, Ker)
    st = _lib().cnn_group_bwd_in(dOut.data_ptr(), Ker.data_ptr(), dIn.data_ptr(),
                                 offsets.data_ptr(), Np, Ng, Nc, Nk, dt, _raw(stream))
    if st:
        _check(st)
    return dIn


def group_bwd_ker(dOut, In, dKer, offsets, rows=None, stream=None):
    """dKer[g] = sum over group g's places p of dOut[p]^T In[rows[p]]: dOut
    [Np, Nk], In [Nt, Nc], dKer [Ng, Nk, Nc]; zeros for an empty group."""
    if not _same(_enter(), dOut, In, dKer, offsets, offsets if rows is None else rows):
        _refuse(dOut=dOut, In=In, dKer=dKer, offsets=offsets, rows=rows)
    Np, Nk = _dims("dOut", dOut, 2)
    Nt, Nc = _dims("In", In, 2)
    Ng = _dims("dKer", dKer, 3)[0]
    _shape("dKer", dKer, Ng, Nk, Nc)
    if rows is None:
        _shape("In", In, Np, Nc)
    _group(offsets, rows, Np, Ng)
    dt = _dtype(dKer, dOut, In)
    st = _lib().cnn_group_bwd_ker(dOut.data_ptr(), In.data_ptr(), dKer.data_ptr(),
                                  offsets.data_ptr(), _ptr(rows), Nt, Np, Ng, Nc, Nk, dt,
                                  _raw(stream))
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
    torch = _torch
    n = i64()
    _check(_lib().cnn_adapt_ws(*_adapt_dims(In, Ker, A, Out), ctypes.byref(n)))
    return torch.empty(n.value, dtype=torch.uint8, device=In.device)


def adapt_fwd(In, Ker, A, B, ids, Out, scales=None, ws=None, stream=None):
    """Out[t] = In[t] Ker^T + scales[a] (In[t] A[a]^T) B[a]^T with a = ids[t]
    (outside [0, Na): no adapter): In [Nt, Nc], Ker [Nk, Nc], A [Na, Nl, Nc],
    B [Na, Nk, Nl], scales [Na] float32 (None: ones).  ws: the tensor that
    ``adapt_workspace`` gives, kept by the caller."""
    if not _same(_enter(), In, Ker, A, B, ids, Out, ids if scales is None else scales,
                 ids if ws is None else ws):
        _refuse(In=In, Ker=Ker, A=A, B=B, ids=ids, Out=Out, scales=scales, ws=ws)
    Nt, Nc, Nk, Na, Nl = _adapt_dims(In, Ker, A, Out)
    _shape("B", B, Na, Nk, Nl)
    _shape("ids", ids, Nt)
    _of(_torch.int32, ids=ids)
    if scales is not None:
        _shape("scales", scales, Na)
        _of(_torch.float32, scales=scales)
    dt = _dtype(Out, In, Ker, A, B)
    st = _lib().cnn_adapt_fwd(In.data_ptr(), Ker.data_ptr(), A.data_ptr(), B.data_ptr(),
                              ids.data_ptr(), _ptr(scales), Out.data_ptr(), Nt, Nc, Nk, Na, Nl, dt,
                              _ptr(ws), 0 if ws is None else ws.numel() * ws.element_size(),
                              _raw(stream))
    if st:
        _check(st)
    return Out
