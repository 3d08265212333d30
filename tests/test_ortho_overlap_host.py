"""Orthogonalised updates refuse arrays that share memory, the workspace and the mask among them, before any CUDA call."""
import ctypes

import pytest

from paper_2007_09835_b200 import binding as B

M, K = 32, 64
COUNT, NEED = M * K, B.rt3d_ortho_workspace(M, K)


def ortho(g=1 << 40, out=1 << 41, ws=1 << 42):
    p = B._ortho_params(5, 1e-7, None)
    return B.lib().rt3d_orthogonalize(g, B.RT3D_F32, K, M, K, ctypes.byref(p), out, K, ws, NEED, None)


def update(w=1 << 40, momentum=1 << 41, g=1 << 42, mask=1 << 43, ws=1 << 44):
    p = B.UpdateParams(0.1, 0.9, 0.0, 1.0, 1, B._ortho_params(5, 1e-7, None))
    return B.lib().rt3d_ortho_update(w, momentum, g, B.RT3D_F32, mask, M, K, ctypes.byref(p), ws, NEED, None)


BYTES = {"g": 4 * COUNT, "out": 2 * COUNT, "w": 4 * COUNT, "momentum": 4 * COUNT, "mask": COUNT, "ws": NEED}


@pytest.mark.parametrize("call,names", [(ortho, ("g", "out", "ws")), (update, ("w", "momentum", "g", "mask", "ws"))])
def test_any_two_arrays(call, names):
    with B.planning():
        assert call() == B.OK
        for a in names:
            for b in names:
                if a == b:
                    continue
                start = 1 << 50
                for at in (start, start + BYTES[a] - 16, start - BYTES[b] + 16):
                    assert call(**{a: start, b: at}) == B.ERR_INVALID_ARG, (a, b, at)
                for at in (start + -(-BYTES[a] // 16) * 16, start - -(-BYTES[b] // 16) * 16):        # side by side
                    assert call(**{a: start, b: at}) == B.OK, (a, b, at)
        assert update(mask=None) == B.OK
