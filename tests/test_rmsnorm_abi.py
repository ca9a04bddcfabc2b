"""RMS norm entry points on a machine without a GPU: every refusal comes before any launch."""
import ctypes

import pytest

from paper_1709_05011_amd import larsconv as lc

FAKE = 0x10000000  # never dereferenced: every call below fails validation first, or has no work
OK = lc.RmsNormDesc(4, 100)


def status(fn, *args, **kw):
    with pytest.raises(lc.LarsConvError) as e:
        fn(*args, stream=0, **kw)
    return e.value.status


def fwd(desc, x=FAKE, r=FAKE, g=FAKE, t=FAKE, y=FAKE, rstd=FAKE):
    return status(lc.rmsnorm_fwd, desc, x, r, g, t, y, rstd)


def q8(desc, x=FAKE, r=FAKE, g=FAKE, t=FAKE, y=FAKE, s=FAKE, group=0):
    return status(lc.rmsnorm_fwd_q8, desc, x, r, g, t, y, s, group)


def bwd(desc, h=FAKE, dy=FAKE, dt=FAKE, g=FAKE, rstd=FAKE, dx=FAKE, dg=FAKE, ws=FAKE, nb=1 << 40, h_ld=0):
    return status(lc.rmsnorm_bwd, desc, h, dy, dt, g, rstd, dx, dg, ws, h_ld, workspace_bytes=nb)


def test_descriptor():
    for call in (fwd, q8, bwd):
        for bad in (lc.RmsNormDesc(-1, 8), lc.RmsNormDesc(4, 0), lc.RmsNormDesc(4, -8), lc.RmsNormDesc(4, (1 << 30) + 1),
                    lc.RmsNormDesc(4, 8, x_ld=7), lc.RmsNormDesc(4, 8, residual_ld=-1), lc.RmsNormDesc(1 << 62, 8),
                    lc.RmsNormDesc(1 << 31, 8, x_ld=1 << 31)):
            assert call(bad) == lc.LC_ERR_SHAPE, (call, bad)
            assert lc.rmsnorm_bwd_workspace_bytes(bad) == 0
        for bad in (lc.RmsNormDesc(4, 8, dtype=2), lc.RmsNormDesc(4, 8, eps=-1e-5), lc.RmsNormDesc(4, 8, eps=float("nan"))):
            assert call(bad) == lc.LC_ERR_UNSUPPORTED, (call, bad)
    L, P = lc.lib(), ctypes.c_void_p(FAKE)
    assert L.rmsnorm_fwd(None, P, P, P, P, P, P, None) == lc.LC_ERR_NULL
    assert L.rmsnorm_bwd_workspace_bytes(None) == 0


def test_pointers():
    for name in ("x", "g", "y"):
        assert fwd(OK, **{name: None}) == lc.LC_ERR_NULL
        assert q8(OK, **{name: None}) == lc.LC_ERR_NULL
    assert q8(OK, s=None) == lc.LC_ERR_NULL
    for name in ("h", "dy", "g", "rstd", "dx", "dg"):
        assert bwd(OK, **{name: None}) == lc.LC_ERR_NULL
        assert bwd(OK, **{name: FAKE + 2}) == lc.LC_ERR_ALIGN
    for name in ("x", "r", "g", "t", "y", "rstd"):
        assert fwd(OK, **{name: FAKE + 2}) == lc.LC_ERR_ALIGN
    half = lc.RmsNormDesc(4, 100, dtype=lc.LC_BF16)
    for name in ("x", "r", "t", "y"):
        assert fwd(half, **{name: FAKE + 1}) == lc.LC_ERR_ALIGN
    assert fwd(half, g=FAKE + 2) == lc.LC_ERR_ALIGN
    assert q8(half, s=FAKE + 2) == lc.LC_ERR_ALIGN
    assert fwd(OK, r=None) == lc.LC_ERR_UNSUPPORTED           # a total without a residual


def test_group_and_workspace():
    for group in (-128, 1, 16, 48, 100, 1024):
        assert q8(OK, group=group) == lc.LC_ERR_UNSUPPORTED
    need = lc.rmsnorm_bwd_workspace_bytes(OK)
    assert need >= 4 * 100 * 4 and need % 256 == 0
    assert bwd(OK, ws=None) == lc.LC_ERR_WORKSPACE
    assert bwd(OK, ws=FAKE + 64) == lc.LC_ERR_WORKSPACE
    assert bwd(OK, nb=need - 1) == lc.LC_ERR_WORKSPACE
    assert bwd(OK, h_ld=99) == lc.LC_ERR_SHAPE


def test_no_rows_is_no_work():
    none = lc.RmsNormDesc(0, 100)
    lc.rmsnorm_fwd(none, None, None, None, None, None, stream=0)
    lc.rmsnorm_fwd_q8(none, None, None, None, None, None, None, 128, stream=0)
    assert lc.rmsnorm_bwd_workspace_bytes(none) == 0
