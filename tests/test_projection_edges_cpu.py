"""What the C entry points of linear and rotary take and refuse at the edge of what they allow, on the host: device pointers are
fakes. Calls that pass the checks of their arguments are given a workspace that is too small, so that none is launched."""
import ctypes

import pytest

import paper_2603_08982_amd as sv

INVALID, WORKSPACE = -1, -2
BF16 = 1


def two(b, n):
    return (ctypes.c_int64 * 2)(b, n)


def linear(B=1, N=100, x=0x10000, w=0x100000, y=0x200000, yst=(1700, 17), residual=None, rst=(1700, 17), ws_bytes=1):
    """17 to 17 features in bf16, x in rows that have to be copied."""
    return sv.load_library().svgear_linear(x, two(1700, 17), w, 17, None, BF16, B, N, 17, 17, 0, None, None, residual,
                                           two(*rst), None, y, two(*yst), 0x300000, ws_bytes, None)


def test_a_residual_in_place_may_differ_where_a_stride_does_not_matter():
    assert linear(residual=0x200000) == WORKSPACE
    assert linear(residual=0x200000, rst=(5, 17)) == WORKSPACE  # one batch entry
    assert linear(residual=0x200000, rst=(1700, 18)) == INVALID
    assert linear(B=7, N=1, residual=0x200000, rst=(1700, 5)) == WORKSPACE  # one token of each
    assert linear(B=7, N=1, residual=0x200000, rst=(1701, 17)) == INVALID
    assert linear(B=2, residual=0x200000, rst=(1701, 17)) == INVALID
