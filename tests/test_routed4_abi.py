"""Argument checks of the router's balance and of the contractions in 4 bits, which
need no GPU: every bad call is refused with its documented status before any HIP
call (the addresses below are never read)."""
import ctypes

import pytest

from paper_2105_13480_amd import cnn

F32, BF16, OBF16 = cnn.CNN_F32, cnn.CNN_BF16, cnn.CNN_BF16_OBF16
NULL, SHAPE, DTYPE, OVERFLOW, ALIAS, UNSUPPORTED = -1, -2, -3, -4, -5, -6
P = [i << 44 for i in range(1, 12)]  # addresses far from each other

# entry point -> (pointers, sizes, what follows the sizes)
CALLS = {
    "cnn_balance": (6, (800, 16, 2, 3), (F32, P[8], 1 << 20, None)),
    "cnn_balance_bwd": (7, (800, 16, 2, 3), (OBF16, 1, None)),
    "cnn_quantize4": (3, (8, 72), (F32, 0, None)),
    "cnn_dequantize4": (3, (8, 72), (BF16, None)),
    "cnn_group_fwd4": (7, (8, 16, 3, 72, 40), (BF16, None)),
    "cnn_group_bwd_in4": (5, (16, 3, 72, 40), (OBF16, None)),
}
OPTIONAL = {"cnn_balance": {2}, "cnn_balance_bwd": {2}, "cnn_group_fwd4": {1, 6}}
WRITTEN = {"cnn_balance": (3, 4, 5), "cnn_balance_bwd": (6,), "cnn_quantize4": (1, 2), "cnn_dequantize4": (2,),
           "cnn_group_fwd4": (4,), "cnn_group_bwd_in4": (3,)}
ROWS = {"cnn_balance": {0}, "cnn_balance_bwd": {0}, "cnn_quantize4": {0}, "cnn_dequantize4": {0},
        "cnn_group_fwd4": {0, 1}, "cnn_group_bwd_in4": {0}}
CODES = {"cnn_quantize4": (1,), "cnn_dequantize4": (0,), "cnn_group_fwd4": (0, 2), "cnn_group_bwd_in4": (1,)}


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


@pytest.mark.parametrize("name", ["cnn_group_fwd4", "cnn_group_bwd_in4"])
def test_fp32_rows_refused(name):
    assert _call(name, rest=(F32, None)) == UNSUPPORTED


@pytest.mark.parametrize("name", CALLS)
def test_overlap_refused(name):
    n = CALLS[name][0]
    for w in WRITTEN[name]:
        for i in range(n):
            if i != w:
                ptrs = P[:n]
                ptrs[w] = ptrs[i]
                assert _call(name, ptrs) == ALIAS, (w, i)


@pytest.mark.parametrize("name", CODES)
def test_codes_off_a_boundary_refused(name):
    for i in CODES[name]:
        for off in (1, 4, 8):
            ptrs = P[:CALLS[name][0]]
            ptrs[i] += off
            assert _call(name, ptrs) == SHAPE, (i, off)
            assert b"aligned" in cnn.lib().cnn_last_error()


def test_limits():
    assert _call("cnn_balance", sizes=(8, 1025, 2, 1)) == OVERFLOW
    assert _call("cnn_balance", sizes=(8, 64, 17, 1)) == OVERFLOW
    assert _call("cnn_balance", sizes=(8, 4, 5, 1)) == SHAPE
    assert _call("cnn_balance", sizes=(8, 4, 2, (1 << 20) + 1)) == OVERFLOW
    for name in ("cnn_balance", "cnn_balance_bwd"):  # sequences without bounds
        ptrs = P[:CALLS[name][0]]
        ptrs[2] = None
        assert _call(name, ptrs) == SHAPE
    assert _call("cnn_quantize4", rest=(F32, 2, None)) == UNSUPPORTED
    assert _call("cnn_quantize4", rest=(F32, -1, None)) == UNSUPPORTED
    assert _call("cnn_group_fwd4", sizes=(8, 16, 65536, 24, 40)) == OVERFLOW
    assert _call("cnn_group_fwd4", ptrs=P[:6] + [None]) == SHAPE
    assert _call("cnn_group_fwd4", sizes=(0, 16, 3, 24, 40)) == SHAPE


def test_more_than_a_launch_holds():
    """2^32 threads, tiles past a grid, and sizes whose product wraps: addresses far
    enough apart that nothing overlaps."""
    L, m = cnn.lib(), (1 << 30) - 1
    Q = [i << 58 for i in range(1, 12)]
    assert L.cnn_quantize4(*Q[:3], 1 << 24, 2048, F32, 0, None) == OVERFLOW
    assert L.cnn_dequantize4(*Q[:3], 1 << 24, 2048, BF16, None) == OVERFLOW
    assert L.cnn_balance_bwd(*Q[:7], 1 << 28, 8, 2, 4, F32, 0, None) == OVERFLOW
    for Nc in (64, 7):
        assert L.cnn_group_fwd4(*Q[:7], m, m, 1, Nc, 600, BF16, None) == OVERFLOW
        assert L.cnn_group_fwd4(Q[0], None, *Q[2:7], m, m, 1, Nc, 600, BF16, None) == OVERFLOW
        assert L.cnn_group_bwd_in4(*Q[:5], m, 1, 600 + Nc, Nc, BF16, None) == OVERFLOW
    for Ng, Nk, Nc in ((64, 1 << 29, 1 << 29), (65535, m, m), (32768, m, m)):
        for ker in (Q[2], None):
            assert L.cnn_group_fwd4(Q[0], None, ker, Q[3], Q[4], Q[5], Q[6], 8, 16, Ng, Nc, Nk, BF16, None) == OVERFLOW
            assert L.cnn_group_bwd_in4(Q[0], ker, Q[2], Q[3], Q[4], 16, Ng, Nc, Nk, BF16, None) == OVERFLOW


def test_workspaces():
    L = cnn.lib()
    n = ctypes.c_int64()
    assert L.cnn_balance_ws(10, 8, 1, ctypes.byref(n)) == 0 and n.value == 0
    assert L.cnn_balance_ws(800, 16, 3, ctypes.byref(n)) == 0 and n.value > 0
    need = n.value
    for ws, have, status in ((None, need, NULL), (P[8], need - 1, SHAPE), (P[8] + 8, need, SHAPE),
                             (P[0] + 16, need, ALIAS)):
        assert _call("cnn_balance", rest=(F32, ws, have, None)) == status
    assert L.cnn_balance_ws(8, 4, 1, None) == NULL
    assert L.cnn_balance_ws(8, 0, 1, ctypes.byref(n)) == SHAPE
    assert L.cnn_balance_ws(8, 4, 0, ctypes.byref(n)) == SHAPE


def test_no_rows_no_launch():
    """Calls that have nothing to do return at once, on a machine without a GPU too."""
    assert _call("cnn_quantize4", sizes=(0, 72)) == 0
    assert _call("cnn_dequantize4", sizes=(0, 72)) == 0
    assert _call("cnn_group_fwd4", sizes=(0, 0, 3, 24, 40)) == 0
    assert _call("cnn_group_bwd_in4", sizes=(0, 3, 24, 40)) == 0
    assert _call("cnn_balance_bwd", sizes=(0, 16, 2, 3)) == 0
