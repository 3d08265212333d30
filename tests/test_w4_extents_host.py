"""Extents whose whole tiles pass 32 bits are refused by every call, and the sizes say so."""
import ctypes

import pytest

from paper_2007_09835_b200 import binding as B

FAKE = 0x10000


@pytest.mark.parametrize("m", [2 ** 31 - 63, 2 ** 31 - 16, 2 ** 31 - 15, 2 ** 31 - 1])
def test_many_filters(m):
    assert B.rt3d_w4_codes_bytes(m, 1) == -1 and B.rt3d_w4_scale_count(m, 64, 32) == -1
    q = B.W4(m, 64, 32, FAKE, FAKE, None)
    x, y = B.Tensor(FAKE, 1, 1, 1, 1, 64, 64, B.RT3D_BF16), B.Tensor(1 << 45, 1, 1, 1, 1, m, 2 ** 31 - 8, B.RT3D_BF16)
    lib = B.lib()
    with B.planning():
        assert lib.rt3d_w4_quantize(FAKE, B.RT3D_F32, 64, ctypes.byref(q), None) == B.ERR_UNSUPPORTED
        assert lib.rt3d_w4_unpack(ctypes.byref(q), B.RT3D_F32, FAKE, 64, None) == B.ERR_UNSUPPORTED
        if m <= 2 ** 31 - 8:
            assert lib.rt3d_linear_w4(ctypes.byref(x), ctypes.byref(q), None, 0, ctypes.byref(y), None) == B.ERR_UNSUPPORTED


def test_the_most_filters():
    assert B.rt3d_w4_codes_bytes(2 ** 31 - 64, 1) == (2 ** 27 - 4) * 512
    q = B.W4(2 ** 31 - 64, 64, 32, FAKE, FAKE, None)
    with B.planning():
        assert B.lib().rt3d_w4_quantize(FAKE, B.RT3D_F32, 64, ctypes.byref(q), None) == B.OK
