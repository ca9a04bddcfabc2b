"""AdamW entry points on a machine without a GPU: every refusal comes before any launch."""
import pytest

from paper_1709_05011_amd import larsconv as lc

FAKE = 0x10000000  # never dereferenced: every call below fails validation first, or has no work


def args(q8=False, g_dtype=lc.LC_F32, numel=(100, 5000), lowp=None, **swap):
    a = {k: [FAKE, FAKE] for k in ("w", "g", "m", "v", "m_scale", "v_scale")} | swap
    if q8:
        return lc.AdamWQ8Args(a["w"], a["g"], a["m"], a["m_scale"], a["v"], a["v_scale"], list(numel), lowp, g_dtype)
    return lc.AdamWArgs(a["w"], a["g"], a["m"], a["v"], list(numel), lowp, g_dtype)


def status(a, q8=False, beta1=0.9, beta2=0.99, eps=1e-8, step=1, grad_scale=None):
    with pytest.raises(lc.LarsConvError) as e:
        if q8:
            lc.adamw_step_q8(a, 1e-3, beta1, beta2, eps, 0.1, step, 7, grad_scale=grad_scale, stream=0)
        else:
            lc.adamw_step(a, 1e-3, beta1, beta2, eps, 0.1, step, grad_scale=grad_scale, stream=0)
    return e.value.status


@pytest.mark.parametrize("q8", [False, True])
def test_refusals(q8):
    a = args(q8)
    for bad in (dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=float("nan")), dict(eps=0.0), dict(eps=-1e-8), dict(step=0), dict(step=-3)):
        assert status(a, q8, **bad) == lc.LC_ERR_UNSUPPORTED, bad
    assert status(args(q8, g_dtype=5), q8) == lc.LC_ERR_UNSUPPORTED
    assert status(args(q8, numel=(100, -1)), q8) == lc.LC_ERR_SHAPE
    assert status(args(q8, numel=(100, (1 << 38) + 1)), q8) == lc.LC_ERR_SHAPE
    assert status(a, q8, grad_scale=FAKE + 2) == lc.LC_ERR_ALIGN
    for name in ("w", "g", "m", "v") + (("m_scale", "v_scale") if q8 else ()):
        assert status(args(q8, **{name: [FAKE, None]}), q8) == lc.LC_ERR_NULL, name
        if not (q8 and name in ("m", "v")):
            assert status(args(q8, **{name: [FAKE, FAKE + 2]}), q8) == lc.LC_ERR_ALIGN, name
    assert status(args(q8, g_dtype=lc.LC_BF16, g=[FAKE, FAKE + 1]), q8) == lc.LC_ERR_ALIGN
    assert status(args(q8, lowp=[None, FAKE + 1]), q8) == lc.LC_ERR_ALIGN


def test_lists_of_the_abi():
    L = lc.lib()
    a = args()
    assert L.adamw_step(-1, a.w, a.g, 0, a.m, a.v, a.numel_arr, 0.1, 0.9, 0.9, 1e-8, 0.0, 1, None, None, None, None) == lc.LC_ERR_SHAPE
    for i in (1, 2, 4, 5, 6):
        call = [2, a.w, a.g, 0, a.m, a.v, a.numel_arr, 0.1, 0.9, 0.9, 1e-8, 0.0, 1, None, None, None, None]
        call[i] = None
        assert L.adamw_step(*call) == lc.LC_ERR_NULL
    b = args(True)
    for i in (4, 5, 6, 7):
        call = [2, b.w, b.g, 0, b.m, b.m_scale, b.v, b.v_scale, b.numel_arr, 0.1, 0.9, 0.9, 1e-8, 0.0, 1, 3, None, None, None, None]
        call[i] = None
        assert L.adamw_step_q8(*call) == lc.LC_ERR_NULL
    with pytest.raises(ValueError):
        lc.adamw_step(a, 0.1, 0.9, 0.9, 1e-8, 0.0, 1, weight_decay_per_tensor=[0.1], stream=0)


def test_nothing_to_do():
    lc.adamw_step(lc.AdamWArgs([], [], [], []), 0.1, 0.9, 0.9, 1e-8, 0.0, 1, stream=0)
    lc.adamw_step_q8(lc.AdamWQ8Args([], [], [], [], [], []), 0.1, 0.9, 0.9, 1e-8, 0.0, 1, 1, stream=0)
    none = [None, None]
    lc.adamw_step(lc.AdamWArgs(none, none, none, none, [0, 0]), 0.1, 0.9, 0.9, 1e-8, 0.0, 1, stream=0)


def test_gradients_of_another_type_than_said():
    import torch
    f, h = torch.zeros(4), torch.zeros(4, dtype=torch.bfloat16)
    for g, kind in ((h, lc.LC_F32), (f, lc.LC_BF16), (f.double(), lc.LC_F32)):
        with pytest.raises(ValueError):
            lc.AdamWArgs([f], [g], [f], [f], g_dtype=kind)
    lc.AdamWArgs([f], [f], [f], [f])
    lc.AdamWArgs([f], [h], [f], [f], g_dtype=lc.LC_BF16)


@pytest.mark.parametrize("scale", [0.37, 1.0, 2.5, 0.0])
def test_a_number_in_place_of_a_pointer(scale):
    """grad_scale is a pointer to one float on the device; a Python float would have become address 0 (no scale at all), 1 or 2."""
    with pytest.raises(TypeError):
        lc.adamw_step(args(), 1e-3, 0.9, 0.99, 1e-8, 0.1, 1, grad_scale=scale, stream=0)
    with pytest.raises(TypeError):
        lc.adamw_step_q8(args(True), 1e-3, 0.9, 0.99, 1e-8, 0.1, 1, 7, grad_scale=scale, stream=0)


@pytest.mark.parametrize("q8", [False, True])
def test_lists_that_pointers_would_misread(q8):
    """Lengths, types, strides, sizes and devices of what the arrays of addresses are made from."""
    import torch
    n = 600
    f32, byte = torch.zeros(n), torch.zeros(n, dtype=torch.uint8)
    state, scale = (byte if q8 else f32), torch.zeros(3)

    def make(**swap):
        a = dict(w=[f32, f32], g=[f32, f32], m=[state, state], v=[state, state], numel=None, w_lowp=[None, torch.zeros(n, dtype=torch.bfloat16)], m_scale=[scale, scale],
                 v_scale=[scale, scale]) | swap
        if q8:
            return lc.AdamWQ8Args(a["w"], a["g"], a["m"], a["m_scale"], a["v"], a["v_scale"], a["numel"], a["w_lowp"])
        return lc.AdamWArgs(a["w"], a["g"], a["m"], a["v"], a["numel"], a["w_lowp"])

    make()
    make(w=[f32, FAKE], numel=[n, n], m=[state, FAKE], w_lowp=None)
    if q8:
        make(m=[byte.view(torch.float8_e4m3fn)] * 2, v=[byte.view(torch.float8_e5m2)] * 2)
    names = ("w", "g", "m", "v", "w_lowp") + (("m_scale", "v_scale") if q8 else ())
    for name in names:
        good = scale if "scale" in name else torch.zeros(n, dtype=torch.bfloat16) if name == "w_lowp" else state if name in "mv" else f32
        fewer = good.clone()[:-1]
        for bad in ([good], [good, good, good], [good, good.double()], [good, torch.zeros(2 * good.numel(), dtype=good.dtype)[::2]], [good, good.to("meta")]) + \
                (() if name == "w" else ([good, fewer],)):
            with pytest.raises(ValueError):
                make(**{name: bad})
    with pytest.raises(ValueError):
        make(numel=[n])
    with pytest.raises(ValueError, match="w"):
        make(numel=[n, n + 1])
    with pytest.raises(ValueError):                              # states of the other width
        make(m=[f32 if q8 else byte] * 2)
    for bad in (torch.ones(2), torch.ones(1, dtype=torch.float64)):
        with pytest.raises(ValueError, match="grad_scale"):
            (lc.adamw_step_q8(make(), 1e-3, 0.9, 0.99, 1e-8, 0.1, 1, 7, grad_scale=bad, stream=0) if q8 else
             lc.adamw_step(make(), 1e-3, 0.9, 0.99, 1e-8, 0.1, 1, grad_scale=bad, stream=0))
