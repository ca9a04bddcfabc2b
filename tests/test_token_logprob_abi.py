"""Token log probability entry points on a machine without a GPU: every refusal comes before any launch."""
import ctypes

import pytest

from paper_1709_05011_amd import larsconv as lc

FAKE = 0x10000000  # never dereferenced: every call below fails validation first, or has no work
ONE, MANY, TOP = lc.TokenDesc(4, 100), lc.TokenDesc(4, 131072), lc.TokenDesc(4, 131072, top=5)


def status(fn, *args, **kw):
    with pytest.raises(lc.LarsConvError) as e:
        fn(*args, stream=0, **kw)
    return e.value.status


def fwd(desc, z=FAKE, t=FAKE, lp=FAKE, ent=FAKE, lse=FAKE, ids=None, top=None, ws=FAKE, nb=1 << 40):
    return status(lc.token_logprob_fwd, desc, z, t, lp, ent, lse, ids, top, ws, workspace_bytes=nb)


def bwd(desc, z=FAKE, t=FAKE, lse=FAKE, ent=FAKE, a=FAKE, b=FAKE, dz=FAKE, ld=0):
    return status(lc.token_logprob_bwd, desc, z, t, lse, ent, a, b, dz, ld)


def test_descriptor():
    for call in (fwd, bwd):
        for bad in (lc.TokenDesc(-1, 8), lc.TokenDesc(4, 0), lc.TokenDesc(4, (1 << 30) + 1), lc.TokenDesc(4, 8, ld=7), lc.TokenDesc(4, 8, ld=-8),
                    lc.TokenDesc(1 << 62, 8), lc.TokenDesc(1 << 31, 8, ld=1 << 31)):
            assert call(bad) == lc.LC_ERR_SHAPE, (call, bad)
            assert lc.token_logprob_workspace_bytes(bad) == 0
        for bad in (lc.TokenDesc(4, 8, dtype=3), lc.TokenDesc(4, 8, top=-1), lc.TokenDesc(4, 8, top=33)):
            assert call(bad) == lc.LC_ERR_UNSUPPORTED, (call, bad)
    P = ctypes.c_void_p(FAKE)
    assert lc.lib().token_logprob_fwd(None, P, P, P, P, P, None, None, P, 0, None) == lc.LC_ERR_NULL
    assert lc.token_logprob_workspace_bytes(lc.TokenDesc(0, 8)) == 0


def test_pointers():
    for name in ("z", "t", "lp"):
        assert fwd(ONE, **{name: None}) == lc.LC_ERR_NULL
    for name in ("z", "t", "lp", "ent", "lse"):
        assert fwd(ONE, **{name: FAKE + 2}) == lc.LC_ERR_ALIGN
    assert fwd(TOP, ids=FAKE) == lc.LC_ERR_NULL and fwd(TOP, top=FAKE) == lc.LC_ERR_NULL
    assert fwd(ONE, ids=FAKE, top=FAKE) == lc.LC_ERR_UNSUPPORTED
    half = lc.TokenDesc(4, 100, dtype=lc.LC_BF16)
    assert fwd(half, z=FAKE + 1) == lc.LC_ERR_ALIGN and bwd(half, dz=FAKE + 1) == lc.LC_ERR_ALIGN
    for name in ("z", "t", "lse", "dz"):
        assert bwd(ONE, **{name: None}) == lc.LC_ERR_NULL
    for name in ("z", "t", "lse", "ent", "a", "b", "dz"):
        assert bwd(ONE, **{name: FAKE + 2}) == lc.LC_ERR_ALIGN
    assert bwd(ONE, a=None, b=None) == lc.LC_ERR_NULL and bwd(ONE, ent=None) == lc.LC_ERR_NULL
    assert bwd(ONE, ld=99) == lc.LC_ERR_SHAPE and bwd(ONE, ld=-100) == lc.LC_ERR_SHAPE


def test_workspace():
    assert lc.token_logprob_workspace_bytes(MANY) % 256 == 0
    assert lc.token_logprob_workspace_bytes(TOP) > lc.token_logprob_workspace_bytes(MANY) > 0
    need = lc.token_logprob_workspace_bytes(MANY)
    assert fwd(MANY, ws=None) == lc.LC_ERR_WORKSPACE
    assert fwd(MANY, ws=FAKE + 128) == lc.LC_ERR_WORKSPACE
    assert fwd(MANY, nb=need - 1) == lc.LC_ERR_WORKSPACE


def test_no_rows_is_no_work():
    lc.token_logprob_fwd(lc.TokenDesc(0, 9), None, None, None, stream=0)
    lc.token_logprob_bwd(lc.TokenDesc(0, 9), None, None, None, None, None, None, None, stream=0)
