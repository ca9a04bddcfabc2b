"""Embedding entry points on a machine without a GPU: every refusal comes before any launch."""
import ctypes

import pytest

from paper_1709_05011_amd import larsconv as lc

FAKE = 0x10000000  # never dereferenced: every call below fails validation first, or has no work
OK = lc.EmbeddingDesc(5000, 100, 24)


def status(fn, *args, **kw):
    with pytest.raises(lc.LarsConvError) as e:
        fn(*args, stream=0, **kw)
    return e.value.status


def fwd(desc, table=FAKE, tokens=FAKE, out=FAKE):
    return status(lc.embedding_fwd, desc, table, tokens, out)


def bwd(desc, tokens=FAKE, dout=FAKE, dtable=FAKE, ws=FAKE, nb=1 << 45, accumulate=False):
    return status(lc.embedding_bwd, desc, tokens, dout, dtable, ws, accumulate, workspace_bytes=nb)


def test_descriptor():
    D = lc.EmbeddingDesc
    for call in (fwd, bwd):
        for bad in (D(-1, 8, 8), D((1 << 25) + 1, 8, 8), D(4, 0, 8), D(4, -1, 8), D(4, 8, 0), D(4, 8, -8), D(4, 8, 8, table_ld=7), D(4, 8, 8, table_ld=-1), D(4, (1 << 30) + 1, 8),
                    D(4, 8, (1 << 30) + 1), D(4, 1 << 30, 8, table_ld=1 << 40)):
            assert call(bad) == lc.LC_ERR_SHAPE, (call, bad)
            assert lc.embedding_bwd_workspace_bytes(bad) == 0
        for bad in (D(4, 8, 8, dtype=2), D(4, 8, 8, table_dtype=-1)):
            assert call(bad) == lc.LC_ERR_UNSUPPORTED, (call, bad)
    assert lc.lib().embedding_fwd(None, *[ctypes.c_void_p(FAKE)] * 3, None) == lc.LC_ERR_NULL


def test_pointers_and_workspace():
    for name in ("table", "tokens", "out"):
        assert fwd(OK, **{name: None}) == lc.LC_ERR_NULL
        assert fwd(OK, **{name: FAKE + 2}) == lc.LC_ERR_ALIGN
    for name in ("tokens", "dout", "dtable"):
        assert bwd(OK, **{name: None}) == lc.LC_ERR_NULL
        assert bwd(OK, **{name: FAKE + 2}) == lc.LC_ERR_ALIGN
    half = lc.EmbeddingDesc(5, 100, 24, table_dtype=lc.LC_BF16, dtype=lc.LC_BF16)
    assert fwd(half, table=FAKE + 1) == lc.LC_ERR_ALIGN and fwd(half, out=FAKE + 1) == lc.LC_ERR_ALIGN and bwd(half, dout=FAKE + 1) == lc.LC_ERR_ALIGN
    for desc in (OK, half):
        need = lc.embedding_bwd_workspace_bytes(desc)
        assert need > 0 and need % 256 == 0
        assert bwd(desc, ws=None) == lc.LC_ERR_WORKSPACE and bwd(desc, ws=FAKE + 64) == lc.LC_ERR_WORKSPACE and bwd(desc, nb=need - 1) == lc.LC_ERR_WORKSPACE


def test_no_rows_is_no_work():
    none = lc.EmbeddingDesc(0, 100, 24)
    lc.embedding_fwd(none, None, None, None, stream=0)
    lc.embedding_bwd(none, None, None, None, None, accumulate=True, stream=0)
    assert bwd(none, dtable=None) == lc.LC_ERR_NULL
    assert lc.embedding_bwd_workspace_bytes(none) == 0
