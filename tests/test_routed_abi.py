"""The routed contractions' argument checks, which need no GPU: every bad call
is refused with its documented status before any HIP call (the addresses
below are never read)."""
import ctypes

import pytest

from paper_2105_13480_amd import cnn

F32, BF16, OBF16 = cnn.CNN_F32, cnn.CNN_BF16, cnn.CNN_BF16_OBF16
NULL, SHAPE, DTYPE, OVERFLOW, ALIAS, UNSUPPORTED = -1, -2, -3, -4, -5, -6
P = [i << 44 for i in range(1, 12)]  # addresses far from each other

# entry point -> (pointers, sizes, what follows the sizes)
CALLS = {
    "cnn_route": (6, (8, 16, 2), (F32, 0, P[8], 1 << 20, None)),
    "cnn_route_bwd": (5, (8, 16, 2), (F32, 1, None)),
    "cnn_combine": (4, (8, 2, 16, 24), (BF16, None)),
    "cnn_combine_bwd": (7, (8, 2, 16, 24), (BF16, None)),
    "cnn_group_fwd": (5, (8, 16, 3, 24, 40), (F32, None)),
    "cnn_group_bwd_in": (4, (16, 3, 24, 40), (BF16, None)),
    "cnn_group_bwd_ker": (5, (8, 16, 3, 24, 40), (OBF16, None)),
    "cnn_adapt_fwd": (7, (200, 24, 40, 3, 8), (OBF16, P[8], 1 << 20, None)),
}
# pointers that may be NULL: weights, and what is asked for only at times
OPTIONAL = {"cnn_combine": {2}, "cnn_combine_bwd": {4, 6}, "cnn_group_fwd": {4}, "cnn_group_bwd_ker": {4},
            "cnn_adapt_fwd": {5}}
# pointers that are written
WRITTEN = {"cnn_route": (1, 2, 3, 4, 5), "cnn_route_bwd": (4,), "cnn_combine": (3,), "cnn_combine_bwd": (5, 6),
           "cnn_group_fwd": (2,), "cnn_group_bwd_in": (2,), "cnn_group_bwd_ker": (2,), "cnn_adapt_fwd": (6,)}
# sizes that may be zero (a call without rows)
ROWS = {"cnn_route": {0}, "cnn_route_bwd": {0}, "cnn_combine": {0, 2}, "cnn_combine_bwd": {0, 2},
        "cnn_group_fwd": {0, 1}, "cnn_group_bwd_in": {0}, "cnn_group_bwd_ker": {0, 1}, "cnn_adapt_fwd": {0}}


def _call(name, ptrs=None, sizes=None, rest=None):
    n, s, r = CALLS[name]
    return getattr(cnn.lib(), name)(*(P[:n] if ptrs is None else ptrs), *(s if sizes is None else sizes),
                                    *(r if rest is None else rest))


@pytest.mark.parametrize("name", CALLS)
def test_null_refused(name):
    for i in range(CALLS[name][0]):
        if i in OPTIONAL.get(name, ()):
            continue
        ptrs = P[:CALLS[name][0]]
        ptrs[i] = None
        assert _call(name, ptrs) == NULL, i
        assert b"non-NULL" in cnn.lib().cnn_last_error()


@pytest.mark.parametrize("name", CALLS)
def test_sizes_refused(name):
    for i in range(len(CALLS[name][1])):
        for value, status in ((-1, {SHAPE}), (0, {SHAPE}), (1 << 40, {OVERFLOW, SHAPE}), (1 << 62, {OVERFLOW, SHAPE})):
            if value == 0 and i in ROWS[name]:
                continue
            sizes = list(CALLS[name][1])
            sizes[i] = value
            assert _call(name, sizes=sizes) in status, (i, value)


@pytest.mark.parametrize("name", CALLS)
def test_types_refused(name):
    for bad in (-1, 3, 77):
        assert _call(name, rest=(bad, *CALLS[name][2][1:])) == DTYPE


@pytest.mark.parametrize("name", CALLS)
def test_overlap_refused(name):
    n = CALLS[name][0]
    for w in WRITTEN[name]:
        for i in range(n):
            if i != w:
                ptrs = P[:n]
                ptrs[w] = ptrs[i] + 4
                assert _call(name, ptrs) == ALIAS, (w, i)


def test_limits():
    assert _call("cnn_route", sizes=(8, 1025, 2)) == OVERFLOW
    assert _call("cnn_route", sizes=(8, 64, 17)) == OVERFLOW
    assert _call("cnn_route", sizes=(8, 4, 5)) == SHAPE
    assert _call("cnn_route", rest=(F32, 2, P[8], 1 << 20, None)) == UNSUPPORTED
    assert _call("cnn_route_bwd", rest=(F32, -1, None)) == UNSUPPORTED
    assert _call("cnn_group_fwd", sizes=(8, 16, 65536, 24, 40)) == OVERFLOW
    assert _call("cnn_adapt_fwd", sizes=(200, 24, 40, 1025, 8)) == OVERFLOW
    # more tiles than a launch holds
    assert _call("cnn_group_fwd", sizes=(8, 1 << 29, 3, 24, 1 << 20)) == OVERFLOW
    # without Rows the rows of In are the places; rows of nothing
    assert _call("cnn_group_fwd", ptrs=P[:4] + [None]) == SHAPE
    assert _call("cnn_group_fwd", sizes=(0, 16, 3, 24, 40)) == SHAPE


def test_workspaces():
    L = cnn.lib()
    n = ctypes.c_int64()
    assert L.cnn_route_ws(1, 8, 2, ctypes.byref(n)) == 0 and n.value == 0
    assert L.cnn_route_ws(100000, 64, 2, ctypes.byref(n)) == 0 and n.value > 0
    need, sizes = n.value, (100000, 64, 2)
    for ws, have, status in ((None, need, NULL), (P[8], need - 1, SHAPE), (P[8] + 8, need, SHAPE)):
        assert _call("cnn_route", sizes=sizes, rest=(F32, 0, ws, have, None)) == status
    assert L.cnn_adapt_ws(200, 24, 40, 3, 8, ctypes.byref(n)) == 0
    need = n.value
    for ws, have, status in ((None, need, NULL), (P[8], need - 1, SHAPE), (P[8] + 4, need, SHAPE),
                             (P[6] + 16, need, ALIAS)):
        assert _call("cnn_adapt_fwd", rest=(OBF16, ws, have, None)) == status
    assert L.cnn_route_ws(8, 4, 2, None) == NULL and L.cnn_adapt_ws(8, 4, 2, 1, 1, None) == NULL
    assert L.cnn_route_ws(8, 0, 2, ctypes.byref(n)) == SHAPE
    assert L.cnn_adapt_ws(8, 4, 2, 1, 0, ctypes.byref(n)) == SHAPE


def test_no_rows_no_launch():
    """Calls that have nothing to do return at once, on a machine without a GPU too."""
    assert _call("cnn_group_fwd", sizes=(0, 0, 3, 24, 40)) == 0
    assert _call("cnn_group_bwd_in", sizes=(0, 3, 24, 40)) == 0
    assert _call("cnn_combine", sizes=(0, 2, 16, 24)) == 0
    assert _call("cnn_combine_bwd", sizes=(0, 2, 0, 24)) == 0
    assert _call("cnn_route_bwd", sizes=(0, 16, 2)) == 0
    assert _call("cnn_adapt_fwd", sizes=(0, 24, 40, 3, 8)) == 0
