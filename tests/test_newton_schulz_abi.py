"""Newton-Schulz and optimizer entry points on a machine without a GPU: every refusal comes before any launch."""
import ctypes

import pytest
import torch

from paper_1709_05011_amd import larsconv as lc

FAKE = 0x10000000  # never dereferenced: every call below fails validation first, or has no work
OK = lc.NewtonSchulzDesc(2, 40, 30)


def status(fn, *args, **kw):
    with pytest.raises(lc.LarsConvError) as e:
        fn(*args, stream=0, **kw)
    return e.value.status


def ns(desc, x=FAKE, y=FAKE, ws=FAKE, nb=1 << 45):
    return status(lc.newton_schulz, desc, x, y, ws, workspace_bytes=nb)


def test_descriptor():
    D = lc.NewtonSchulzDesc
    for bad in (D(-1, 8, 8), D(1, 0, 8), D(1, 8, 0), D(1, -3, 8), D(1, 65537, 8), D(1, 8, 65537), D(1, 8, 8, ld=7), D(1, 8, 8, ld=-1), D(1 << 30, 60000, 8, ld=1 << 39)):
        assert ns(bad) == lc.LC_ERR_SHAPE, bad
        assert lc.newton_schulz_workspace_bytes(bad) == 0
    for bad in (D(1, 8, 8, dtype=2), D(1, 8, 8, iterations=0), D(1, 8, 8, iterations=65), D(1, 8, 8, eps=-1.0), D(1, 8, 8, eps=float("nan"))):
        assert ns(bad) == lc.LC_ERR_UNSUPPORTED, bad
    assert lc.lib().newton_schulz(None, ctypes.c_void_p(FAKE), ctypes.c_void_p(FAKE), ctypes.c_void_p(FAKE), 1 << 40, None) == lc.LC_ERR_NULL
    lc.newton_schulz(D(0, 8, 8), None, None, None, stream=0)


def test_pointers_and_workspace():
    assert ns(OK, x=None) == lc.LC_ERR_NULL and ns(OK, y=None) == lc.LC_ERR_NULL
    assert ns(OK, x=FAKE + 2) == lc.LC_ERR_ALIGN and ns(OK, y=FAKE + 2) == lc.LC_ERR_ALIGN
    need = lc.newton_schulz_workspace_bytes(OK)
    assert need % 256 == 0 and need >= 2 * (8 * 64 * 32 + 8 * 32 * 32)
    assert ns(OK, ws=None) == lc.LC_ERR_WORKSPACE and ns(OK, ws=FAKE + 128) == lc.LC_ERR_WORKSPACE and ns(OK, nb=need - 1) == lc.LC_ERR_WORKSPACE


class Plain:
    """A list of addresses."""

    def __init__(self, shapes, **other):
        self.shapes, self.other = shapes, other

    def call(self, momentum=0.95, iterations=5, eps=1e-7, ws=FAKE, nb=1 << 45, g_dtype=lc.LC_F32, grad_scale=None):
        lists = {k: self.other.get(k, [FAKE] * len(self.shapes)) for k in ("w", "g", "m")}
        args = lc.MuonArgs(lists["w"], lists["g"], lists["m"], w_lowp=self.other.get("w_lowp"), g_dtype=g_dtype, shapes=self.shapes)
        return status(lc.muon_step, args, 0.02, momentum, 0.1, ws, iterations=iterations, eps=eps, grad_scale=grad_scale, workspace_bytes=nb)


def test_lists():
    one = [(8, 9)]
    assert Plain([(8, 65537)]).call() == lc.LC_ERR_SHAPE and Plain([(-1, 8)]).call() == lc.LC_ERR_SHAPE
    for name in ("w", "g", "m"):
        assert Plain(one, **{name: [None]}).call() == lc.LC_ERR_NULL
        assert Plain(one, **{name: [FAKE + 2]}).call() == lc.LC_ERR_ALIGN
    assert Plain(one, g=[FAKE + 1]).call(g_dtype=lc.LC_BF16) == lc.LC_ERR_ALIGN
    assert Plain(one, w_lowp=[FAKE + 1]).call() == lc.LC_ERR_ALIGN
    assert Plain(one).call(grad_scale=FAKE + 2) == lc.LC_ERR_ALIGN
    for bad in (dict(momentum=1.0), dict(momentum=-0.1), dict(momentum=float("nan")), dict(iterations=0), dict(iterations=65), dict(eps=-1.0), dict(g_dtype=3)):
        assert Plain(one).call(**bad) == lc.LC_ERR_UNSUPPORTED, bad
    args = lc.MuonArgs([FAKE], [FAKE], [FAKE], shapes=one)
    need = lc.muon_workspace_bytes(args)
    assert Plain(one).call(ws=None) == lc.LC_ERR_WORKSPACE and Plain(one).call(nb=need - 1) == lc.LC_ERR_WORKSPACE and Plain(one).call(ws=FAKE + 64) == lc.LC_ERR_WORKSPACE
    empty = lc.MuonArgs([FAKE] * 2, [FAKE] * 2, [FAKE] * 2, shapes=[(0, 4), (5, 0)])
    lc.muon_step(empty, 0.02, 0.95, 0.1, None, stream=0)
    lc.muon_step(lc.MuonArgs([], [], []), 0.02, 0.95, 0.1, None, stream=0)


def test_workspace_is_shared_by_groups():
    of = lambda *shapes: lc.muon_workspace_bytes(lc.MuonArgs([FAKE] * len(shapes), [FAKE] * len(shapes), [FAKE] * len(shapes), shapes=shapes))
    single = of((4096, 4096))
    assert 16 * 4096 * 4096 <= single <= 16 * 4096 * 4096 + 16384
    assert of(*[(4096, 4096)] * 40) == 7 * single <= 2 << 30                          # as many as 2 GiB hold
    assert of(*[(64, 64)] * 200) == of(*[(64, 64)] * 64)
    assert of((65536, 65536)) > 2 << 30
    assert of((100, 300), (4096, 4096)) == of((4096, 4096), (100, 300))


def test_tensors_are_checked_where_their_addresses_are_taken():
    w = [torch.zeros(4, 6)]
    for bad in (dict(g=[torch.zeros(4, 6, dtype=torch.bfloat16)]), dict(m=[torch.zeros(4, 6, dtype=torch.float64)]), dict(g=[torch.zeros(6, 4).T]), dict(m=[torch.zeros(4, 5)]),
                dict(g=[]), dict(w_lowp=[torch.zeros(4, 6)]), dict(shapes=[(4, 6), (1, 1)])):
        with pytest.raises(ValueError):
            lc.MuonArgs(**({"w": w, "g": [torch.zeros(4, 6)], "m": [torch.zeros(4, 6)]} | bad))
    with pytest.raises(ValueError):
        lc.muon_step(lc.MuonArgs(w, [torch.zeros(4, 6)], [torch.zeros(4, 6)]), 0.1, 0.9, 0.0, None, scale_per_tensor=[1.0, 2.0], stream=0)
