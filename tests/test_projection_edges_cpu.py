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


def rotary(B=1, H=3, N=30, dst=0x100000, dst_st=(5760, 1920, 64), src_st=(5760, 1920, 64), back=False):
    """In place, 64 elements a head, with a norm over the token; the backward pass wants dweight and has too little room for it. The
    forward pass has no workspace: only what it refuses can be asked."""
    lib = sv.load_library()
    ptr = lambda p: (ctypes.c_void_p * 1)(p)
    st = lambda s: (ctypes.c_int64 * 3)(*s)
    places = (0x10000, (ctypes.c_int * 3)(10, 11, 11), (ctypes.c_int64 * 3)(2, 3, 5), 0, None, 0, 2, 1e-6)
    if not back:
        return lib.svgear_rotary(1, ptr(0x100000), st(src_st), ptr(dst), st(dst_st), None, BF16, B, H, N, 0, 64, *places, None)
    return lib.svgear_rotary_backward(1, ptr(0x100000), st(src_st), ptr(0x400000), st(src_st), ptr(dst), st(dst_st), None, ptr(0x500000), BF16, B, H,
                                      N, 0, 64, *places, 0x300000, 1, None)


def test_rotary_in_place_at_other_strides():
    for back in (False, True):
        assert rotary(dst_st=(5760, 1920, 72), back=back) == INVALID
        assert rotary(dst_st=(5760, 1928, 64), back=back) == INVALID
        assert rotary(B=2, N=10, dst_st=(5768, 1920, 64), back=back) == INVALID
    assert rotary(back=True) == WORKSPACE
    assert rotary(dst_st=(7, 1920, 64), back=True) == WORKSPACE                                     # one batch entry
    assert rotary(H=1, src_st=(5760, 5, 64), dst_st=(9, 1920, 64), back=True) == WORKSPACE            # and one head
    assert rotary(N=1, src_st=(64, 1920, 3), dst_st=(64, 1920, 72), back=True) == WORKSPACE           # one token


def test_rotary_refuses_gradients_of_weights_over_other_outputs():
    lib = sv.load_library()
    pair = lambda *p: (ctypes.c_void_p * 2)(*p)
    st = (ctypes.c_int64 * 6)(*(2 * [5760, 1920, 64]))
    places = (0x10000, (ctypes.c_int * 3)(10, 11, 11), (ctypes.c_int64 * 3)(2, 3, 5), 0, None, 0, 2, 1e-6)
    dy, src, dx, weight = (0x100000, 0x200000), (0x300000, 0x400000), (0x500000, 0x600000), (0x700000, 0x800000)

    def call(*dweight):
        return lib.svgear_rotary_backward(2, pair(*dy), st, pair(*src), st, pair(*dx), st, pair(*weight), pair(*dweight), BF16, 1, 3, 30, 0, 64,
                                          *places, 0x900000, 1, None)

    assert call(0xa00000, 0xb00000) == call(0xa00000, None) == call(None, 0xb00000) == WORKSPACE
    assert call(0xa00000, 0xa00000) == INVALID
    for other in dx:
        assert call(other, 0xb00000) == INVALID and call(0xa00000, other) == INVALID, hex(other)
