"""4-bit weights: sizes and refusals, all before any CUDA call."""
import ctypes

import pytest

from paper_2007_09835_b200 import binding as B

FAKE = 0x10000     # a 16-byte aligned, never dereferenced address


def w4(m=32, k=64, group=32, codes=FAKE, scales=FAKE, zeros=None):
    return B.W4(m, k, group, codes, scales, zeros)


def test_sizes():
    assert B.rt3d_w4_codes_bytes(1, 1) == 512
    assert B.rt3d_w4_codes_bytes(17, 65) == 4 * 512
    assert B.rt3d_w4_codes_bytes(4096, 8192) == 4096 * 8192 // 2
    assert B.rt3d_w4_scale_count(17, 65, 32) == 32 * 3
    assert B.rt3d_w4_scale_count(16, 128, 128) == 16
    for m, k in ((0, 64), (16, 0), (-1, 64), (2 ** 31 - 1, 2 ** 31 - 1), (1, 2 ** 30 + 1)):
        assert B.rt3d_w4_codes_bytes(m, k) == -1 and B.rt3d_w4_scale_count(m, k, 32) == -1
    for group in (0, 16, 48, 256, -32):
        assert B.rt3d_w4_scale_count(16, 64, group) == -1


BAD = [dict(m=0), dict(k=0), dict(m=-5), dict(group=16), dict(group=33), dict(codes=None), dict(scales=None), dict(codes=FAKE + 8),
       dict(scales=FAKE + 4), dict(zeros=FAKE + 2)]


@pytest.mark.parametrize("bad", BAD)
def test_bad_descriptors(bad):
    q = w4(**bad)
    x, y = B.Tensor(FAKE, 1, 1, 1, 1, 64, 64, B.RT3D_BF16), B.Tensor(FAKE + (1 << 20), 1, 1, 1, 1, 32, 32, B.RT3D_BF16)
    lib = B.lib()
    assert lib.rt3d_w4_quantize(FAKE, B.RT3D_F32, 64, ctypes.byref(q), None) == B.ERR_INVALID_ARG
    assert lib.rt3d_w4_unpack(ctypes.byref(q), B.RT3D_F32, FAKE, 64, None) == B.ERR_INVALID_ARG
    assert lib.rt3d_linear_w4(ctypes.byref(x), ctypes.byref(q), None, 0, ctypes.byref(y), None) == B.ERR_INVALID_ARG


def test_bad_matrices():
    lib, q = B.lib(), w4()
    for ptr, dtype, pitch in ((None, B.RT3D_F32, 64), (FAKE, 2, 64), (FAKE, -1, 64), (FAKE, B.RT3D_F32, 63), (FAKE, B.RT3D_F32, 0),
                              (FAKE + 2, B.RT3D_F32, 64), (FAKE + 1, B.RT3D_BF16, 64)):
        assert lib.rt3d_w4_quantize(ptr, dtype, pitch, ctypes.byref(q), None) == B.ERR_INVALID_ARG
        assert lib.rt3d_w4_unpack(ctypes.byref(q), dtype, ptr, pitch, None) == B.ERR_INVALID_ARG
    assert lib.rt3d_w4_quantize(FAKE, B.RT3D_F32, 64, None, None) == B.ERR_INVALID_ARG


def test_bad_products():
    lib, q = B.lib(), w4()

    def call(x, y, q=q):
        return lib.rt3d_linear_w4(ctypes.byref(x), ctypes.byref(q), None, 0, ctypes.byref(y), None)

    def t(c, cs=None, dtype=B.RT3D_BF16, data=FAKE, n=2):
        return B.Tensor(data, n, 1, 1, 1, c, c if cs is None else cs, dtype)

    far = FAKE + (1 << 20)
    assert call(t(64), t(32, data=far, n=3)) == B.ERR_SHAPE                 # another number of rows
    assert call(t(56), t(32, data=far)) == B.ERR_SHAPE                      # inputs != k
    assert call(t(64), t(24, data=far)) == B.ERR_SHAPE                      # outputs != m
    assert call(t(64), t(32, data=far, dtype=B.RT3D_F32)) == B.ERR_SHAPE    # another type
    assert call(t(64), t(32)) == B.ERR_INVALID_ARG                          # x and y overlap
    assert call(t(64, data=FAKE + 2), t(32, data=far)) == B.ERR_INVALID_ARG
    assert call(t(64, cs=68), t(32, data=far)) == B.ERR_INVALID_ARG         # pitch not a multiple of 8
    assert call(t(64, data=0), t(32, data=far)) == B.ERR_INVALID_ARG
    big = B.Tensor(FAKE, 1 << 16, 1 << 16, 1, 1, 64, 64, B.RT3D_BF16)
    assert call(big, B.Tensor(1 << 45, 1 << 16, 1 << 16, 1, 1, 32, 32, B.RT3D_BF16)) == B.ERR_UNSUPPORTED
    wrap = [B.Tensor(at, 1 << 30, 1 << 30, 1 << 30, 1 << 30, c, c, B.RT3D_BF16) for at, c in ((FAKE, 64), (1 << 45, 32))]
    assert call(*wrap) == B.ERR_UNSUPPORTED                                              # extents whose product passes 64 bits


def test_a_call_of_a_sequence_needs_its_weights():
    lib = B.lib()
    c = B.Call(kind=B.CALL_LINEAR_W4, x=B.Tensor(FAKE, 1, 1, 1, 1, 64, 64, B.RT3D_BF16))
    streams, failed = (ctypes.c_void_p * 1)(None), ctypes.c_int32()
    assert lib.rt3d_run_calls(ctypes.byref(c), 1, streams, 1, ctypes.byref(failed)) == B.ERR_INVALID_ARG and failed.value == 0
