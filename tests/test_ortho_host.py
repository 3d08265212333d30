"""Orthogonalised updates: sizes and refusals, all before any CUDA call."""
import ctypes

import pytest

from paper_2007_09835_b200 import binding as B

FAKE = 0x10000


def ortho(g=FAKE, dtype=B.RT3D_F32, g_pitch=64, m=32, k=64, out=1 << 40, out_pitch=64, ws=1 << 41, size=None, **kw):
    p = B._ortho_params(kw.get("steps", 5), kw.get("eps", 1e-7), kw.get("coefs"))
    size = max(0, B.rt3d_ortho_workspace(m, k)) if size is None else size
    return B.lib().rt3d_orthogonalize(g, dtype, g_pitch, m, k, ctypes.byref(p), out, out_pitch, ws, size, None)


def update(w=FAKE, momentum=1 << 40, g=1 << 41, dtype=B.RT3D_F32, mask=None, m=32, k=64, ws=1 << 42, size=None, lr=0.1, mu=0.9, decay=0.0,
           scale=1.0, **kw):
    p = B.UpdateParams(lr, mu, decay, scale, 1, B._ortho_params(kw.get("steps", 5), kw.get("eps", 1e-7), kw.get("coefs")))
    size = max(0, B.rt3d_ortho_workspace(m, k)) if size is None else size
    return B.lib().rt3d_ortho_update(w, momentum, g, dtype, mask, m, k, ctypes.byref(p), ws, size, None)


def test_workspace_sizes():
    for m, k in ((0, 4), (4, 0), (-1, 4), (1 << 30, 1 << 30)):
        assert B.rt3d_ortho_workspace(m, k) == -1
    assert 0 < B.rt3d_ortho_workspace(1, 1) < B.rt3d_ortho_workspace(512, 13824)
    assert B.rt3d_ortho_workspace(576, 64) == B.rt3d_ortho_workspace(64, 576)


INF, NAN = float("inf"), float("nan")
FLAT = [(1.0, 0.0, 0.0)]


@pytest.mark.parametrize("call", [ortho, update])
def test_bad_arguments(call):
    assert call(g=None) == B.ERR_INVALID_ARG
    assert call(g=(1 << 41) + 2) == B.ERR_INVALID_ARG
    assert call(dtype=2) == B.ERR_INVALID_ARG
    assert call(m=0) == B.ERR_INVALID_ARG and call(k=0) == B.ERR_INVALID_ARG
    assert call(ws=None) == B.ERR_INVALID_ARG and call(ws=(1 << 41) + 8) == B.ERR_INVALID_ARG
    assert call(size=B.rt3d_ortho_workspace(32, 64) - 1) == B.ERR_WORKSPACE and call(size=0) == B.ERR_WORKSPACE
    for steps in (0, -1, 17):
        assert call(steps=steps, coefs=FLAT * steps if steps > 0 else None) == B.ERR_INVALID_ARG
    for eps in (0.0, -1.0, INF, NAN):
        assert call(eps=eps) == B.ERR_INVALID_ARG
    for coefs in ([(NAN, 0, 0)], [(1, INF, 0)], [(1, 0, -INF)]):
        assert call(steps=1, coefs=coefs) == B.ERR_INVALID_ARG


@pytest.mark.parametrize("call", [ortho, update])
@pytest.mark.parametrize("coefs", [
    [(2.0, 0.0, 0.0)],                                  # doubles the largest singular value
    [(51.0, -98.0, 48.0)],                              # 51 at 0
    [(1.5, 0.0, 0.0), (1.5, 0.0, 0.0)],                 # 1.5, then 2.25
    [(0.0, 0.0, 5.0)],
    [(60.0, -60.0, 0.0)],                               # the most lies between the ends
    [(6.0, -5.9, 0.0)],
])
def test_coefficients_that_leave_the_range(call, coefs):
    assert call(steps=len(coefs), coefs=coefs) == B.ERR_UNSUPPORTED


def test_matrices_that_overlap_or_are_too_narrow():
    assert ortho(g_pitch=63) == B.ERR_INVALID_ARG and ortho(out_pitch=63) == B.ERR_INVALID_ARG
    assert ortho(out=None) == B.ERR_INVALID_ARG and ortho(out=(1 << 40) + 1) == B.ERR_INVALID_ARG
    assert ortho(out=FAKE) == B.ERR_INVALID_ARG and ortho(out=FAKE + 4 * (31 * 64 + 63)) == B.ERR_INVALID_ARG


def test_bad_updates():
    assert update(w=None) == B.ERR_INVALID_ARG and update(momentum=None) == B.ERR_INVALID_ARG
    assert update(w=FAKE + 2) == B.ERR_INVALID_ARG and update(momentum=FAKE + 1) == B.ERR_INVALID_ARG
    for name in ("lr", "mu", "decay", "scale"):
        for v in (INF, NAN):
            assert update(**{name: v}) == B.ERR_INVALID_ARG
    assert B.lib().rt3d_ortho_update(FAKE, 1 << 40, 1 << 41, B.RT3D_F32, None, 32, 64, None, 1 << 42, 1 << 30, None) == B.ERR_INVALID_ARG
    assert update(momentum=FAKE) == B.ERR_INVALID_ARG                       # w and momentum, w and g in the same place
    assert update(g=FAKE) == B.ERR_INVALID_ARG
