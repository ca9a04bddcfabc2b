"""GPU parity of the layer norm and its gradient against oracle/token_model_ops.py in float64.

Tolerances count roundings of u = 2^-24 (fp32): a sum over c values in a block's order takes at most c/1024 + 32 of them, deviations, a root, products and the last sum 8 more, hence
k = c/1024 + 64.  A sum of deviations is off by k u of their mean magnitude, which the inverse deviation takes to at most 1: |y - want| <= k u (|n gamma| + |gamma| + |beta|), and
half a step, 2^-8, where y is stored as bf16."""
import numpy as np
import pytest
import torch

from oracle import token_model_ops as ops
from oracle.token_ops import bf16
from paper_1709_05011_amd import larsconv as lc
from paper_1709_05011_amd import synth

import gpu_util as gu

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = {"f32": (lc.LC_F32, torch.float32, 0.0), "bf16": (lc.LC_BF16, torch.bfloat16, 2.0 ** -8)}
# one column to rows beyond a block's registers, odd widths, several rows of a wave, rows beyond the blocks of the backward pass
SHAPES = [(1, 1), (1, 8), (3, 7), (5, 64), (2, 2048), (3, 2049), (4, 4096), (7, 4101), (2, 8192), (2, 8197), (1, 16384), (2, 16385), (2, 20001), (1500, 96), (2100, 33), (300, 256)]


def k_of(c):
    return (c / 1024 + 64) * U


def rows_of(rows, c, seed, dtype, pad=0, offset=0, std=1.0, mean=0.0):
    whole = torch.full((rows * (c + pad) + offset,), float("nan"), dtype=dtype, device=gu.DEV)
    view = whole[offset:].view(rows, c + pad)[:, :c]
    view.copy_(torch.from_numpy(synth.normal((rows, c), seed, std=std, mean=mean)))
    return view, view.double().cpu().numpy()


def store_of(kind):
    return (lambda v: bf16(v.astype(np.float32))) if kind == "bf16" else (lambda v: v.astype(np.float32).astype(np.float64))


def f64(t):
    return t.double().cpu().numpy()


def check_forward(kind, c, h64, gamma, beta, eps, y, mean, rstd):
    half = TYPES[kind][2]
    _, want_mean, want_rstd, n, want = ops.layernorm(h64, None, f64(gamma), None if beta is None else f64(beta), eps)
    spread = np.mean(np.abs(h64 - want_mean[:, None]), axis=1)
    assert np.all(np.abs(f64(mean) - want_mean) <= k_of(c) * spread + U * np.abs(want_mean))
    assert np.all(np.abs(f64(rstd) - want_rstd) <= k_of(c) * want_rstd)
    g, b = np.abs(f64(gamma)), 0.0 if beta is None else np.abs(f64(beta))
    assert np.all(np.abs(f64(y) - want) <= half * (1 + half) * np.abs(want) + k_of(c) * (1 + half) * (np.abs(n) * g + g + b))


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rows,c", SHAPES)
@pytest.mark.parametrize("residual,pad,offset,shift", [(True, 0, 0, True), (False, 0, 0, False), (True, 5, 1, False), (False, 3, 1, True)])
def test_forward(kind, rows, c, residual, pad, offset, shift):
    dtype, t, _ = TYPES[kind]
    x, x64 = rows_of(rows, c, 1, t, pad, offset, mean=0.5)
    r, r64 = rows_of(rows, c, 2, t, 2 * pad, offset, std=3.0) if residual else (None, None)
    gamma, beta = gu.dev(1 + synth.normal((c,), 3, std=0.3)), gu.dev(synth.normal((c,), 4)) if shift else None
    total, check_t = gu.guarded((rows, c), t, offset=offset * 4)
    y, check_y = gu.guarded((rows, c), t, offset=offset * 4)
    mean, check_m = gu.guarded((rows,), torch.float32)
    rstd, check_r = gu.guarded((rows,), torch.float32)
    d = lc.LayerNormDesc(rows, c, x_ld=c + pad, residual_ld=c + 2 * pad, eps=1e-5, dtype=dtype)
    lc.layernorm_fwd(d, x, r, gamma, beta, total if residual else None, y, mean, rstd)
    torch.cuda.synchronize()
    for check in (check_t, check_y, check_m, check_r):
        check()
    h64 = x64 if r is None else store_of(kind)(x64 + r64)
    if residual:
        assert np.array_equal(f64(total), h64)
    check_forward(kind, c, h64, gamma, beta, float(np.float32(1e-5)), y, mean, rstd)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rows,c", SHAPES)
@pytest.mark.parametrize("joined,pad,shift", [(True, 0, True), (False, 3, True), (True, 1, False)])
def test_backward(kind, rows, c, joined, pad, shift):
    dtype, t, half = TYPES[kind]
    h, h64 = rows_of(rows, c, 7, t, pad, std=2.0, mean=0.7)
    dy, dy64 = rows_of(rows, c, 8, t, 0, pad, std=0.1, mean=0.02)
    dt, dt64 = rows_of(rows, c, 9, t, 0, pad, std=0.1) if joined else (None, None)
    gamma = gu.dev(1 + synth.normal((c,), 10, std=0.3))
    mean = gu.dev(np.mean(h64, axis=1).astype(np.float32))
    rstd = gu.dev((1 / np.sqrt(np.var(h64, axis=1) + 1e-5)).astype(np.float32))
    dx, check_x = gu.guarded((rows, c), t)
    dg, check_g = gu.guarded((c,), torch.float32)
    db, check_b = gu.guarded((c,), torch.float32)
    d = lc.LayerNormDesc(rows, c, dtype=dtype)
    ws = gu.workspace(lc.layernorm_bwd_workspace_bytes(d))
    lc.layernorm_bwd(d, h, dy, dt, gamma, mean, rstd, dx, dg, db if shift else None, ws, h_ld=c + pad)
    torch.cuda.synchronize()
    for check in (check_x, check_g, check_b):
        check()
    m64, r64, g64 = f64(mean), f64(rstd), f64(gamma)
    want, want_g, want_b = ops.layernorm_bwd(h64, m64, r64, g64, dy64, dt64)
    n, a = np.abs((h64 - m64[:, None]) * r64[:, None]), np.abs(dy64 * g64)
    parts = r64[:, None] * (a + np.mean(a, axis=1, keepdims=True) + n * np.mean(a * n, axis=1, keepdims=True)) + (0 if dt is None else np.abs(dt64))
    assert np.all(np.abs(f64(dx) - want) <= half * (1 + half) * np.abs(want) + (k_of(c) * (1 + half)) * parts)
    assert np.all(np.abs(f64(dg) - want_g) <= (rows + 64) * U * np.sum(np.abs(dy64) * n, axis=0))
    if shift:
        assert np.all(np.abs(f64(db) - want_b) <= (rows + 64) * U * np.sum(np.abs(dy64), axis=0))
    else:
        assert bool(torch.isnan(db).all())


def test_the_gradient_against_differences():
    """Central differences of the float64 sum of y * dy through the kernel's own forward pass, fp32: a step of 2^-6 keeps its rounding under 1e-3."""
    rows, c, e = 2, 24, 2.0 ** -6
    x, dy = synth.normal((rows, c), 11), synth.normal((rows, c), 12)
    gamma, beta = gu.dev(1 + synth.normal((c,), 13, std=0.3)), gu.dev(synth.normal((c,), 14))
    d = lc.LayerNormDesc(rows, c, eps=1e-3)
    y, mean, rstd = torch.empty((rows, c), device=gu.DEV), torch.empty(rows, device=gu.DEV), torch.empty(rows, device=gu.DEV)

    def forward(a, g=gamma, b=beta):
        lc.layernorm_fwd(d, gu.dev(a.astype(np.float32)), None, g, b, None, y, mean, rstd)
        return float(np.sum(f64(y) * dy))

    forward(x)
    dx, dg, db = torch.empty((rows, c), device=gu.DEV), torch.empty(c, device=gu.DEV), torch.empty(c, device=gu.DEV)
    lc.layernorm_bwd(d, gu.dev(x), gu.dev(dy), None, gamma, mean, rstd, dx, dg, db, gu.workspace(lc.layernorm_bwd_workspace_bytes(d)))
    got = f64(dx)
    for i, j in [(0, 0), (0, 23), (1, 5), (1, 12)]:
        up, down = x.copy(), x.copy()
        up[i, j] += np.float32(e)
        down[i, j] -= np.float32(e)
        numeric = (forward(up) - forward(down)) / float(up[i, j].astype(np.float64) - down[i, j].astype(np.float64))
        assert abs(numeric - got[i, j]) < 2e-3 * max(1.0, abs(got[i, j]))
    for j in (0, 11, 23):
        for of, grad in ((0, dg), (1, db)):
            up, down = [gamma.clone(), beta.clone()], [gamma.clone(), beta.clone()]
            up[of][j] += e
            down[of][j] -= e
            numeric = (forward(x, *up) - forward(x, *down)) / float(up[of][j].double() - down[of][j].double())
            assert abs(numeric - float(grad[j])) < 2e-3 * max(1.0, abs(float(grad[j])))


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("c", [96, 5000, 17000])
def test_total_in_the_residuals_own_buffer(kind, c):
    dtype, t, _ = TYPES[kind]
    x, _ = rows_of(3, c, 14, t)
    r, _ = rows_of(3, c, 15, t)
    gamma, d = torch.ones(c, device=gu.DEV), lc.LayerNormDesc(3, c, dtype=dtype)
    want_t, want_y, y = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    lc.layernorm_fwd(d, x, r, gamma, None, want_t, want_y)
    lc.layernorm_fwd(d, x, r, gamma, None, r, y)
    torch.cuda.synchronize()
    assert torch.equal(r, want_t) and torch.equal(y, want_y)


@pytest.mark.parametrize("c", [8, 33, 256, 2048, 9001, 20000])
@pytest.mark.parametrize("size", [1e-30, 1e-22, 1e19, 1e38])
def test_rows_beyond_the_range_of_squares(c, size):
    """eps 0: the statistics are those of the values, whatever their size.  (Deviations of some 1e38 leave fp32 by themselves.)"""
    base = synth.normal((300, c), 16, mean=0.4)
    base = np.clip(base, -3, 3)
    x = gu.dev((base * np.float32(size)).astype(np.float32))
    gamma, y, mean, rstd = torch.ones(c, device=gu.DEV), torch.empty((300, c), device=gu.DEV), torch.empty(300, device=gu.DEV), torch.empty(300, device=gu.DEV)
    lc.layernorm_fwd(lc.LayerNormDesc(300, c, eps=0.0), x, None, gamma, None, None, y, mean, rstd)
    torch.cuda.synchronize()
    x64 = f64(x)
    _, _, want_rstd, n, want = ops.layernorm(x64, None, np.ones(c), None, 0.0)
    assert np.all(np.abs(f64(y) - want) <= k_of(c) * (np.abs(n) + 1))
    normal = want_rstd >= 2.0 ** -126
    assert np.all(np.abs(f64(rstd) - want_rstd)[normal] <= (k_of(c) * want_rstd)[normal])


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("c", [64, 200, 4096, 20000])
def test_a_mean_far_from_zero(kind, c):
    dtype, t, _ = TYPES[kind]
    x, x64 = rows_of(4, c, 17, t, mean=1000.0)
    gamma, beta = gu.dev(1 + synth.normal((c,), 18, std=0.3)), gu.dev(synth.normal((c,), 19))
    y, mean, rstd = torch.empty((4, c), dtype=t, device=gu.DEV), torch.empty(4, device=gu.DEV), torch.empty(4, device=gu.DEV)
    lc.layernorm_fwd(lc.LayerNormDesc(4, c, dtype=dtype), x, None, gamma, beta, None, y, mean, rstd)
    torch.cuda.synchronize()
    check_forward(kind, c, x64, gamma, beta, float(np.float32(1e-5)), y, mean, rstd)


@pytest.mark.parametrize("c", [64, 200, 4096, 20000])
def test_constant_rows_and_rows_that_hold_no_numbers(c):
    x = synth.normal((8, c), 20)
    x[1], x[2] = 0.0, 7.25
    x[4, c // 2], x[6, 3] = np.nan, np.inf
    xd, gamma, beta = gu.dev(x), torch.ones(c, device=gu.DEV), gu.dev(synth.normal((c,), 21))
    y, mean, rstd = torch.empty((8, c), device=gu.DEV), torch.empty(8, device=gu.DEV), torch.empty(8, device=gu.DEV)
    lc.layernorm_fwd(lc.LayerNormDesc(8, c), xd, None, gamma, beta, None, y, mean, rstd)
    torch.cuda.synchronize()
    got = f64(y)
    assert np.all(np.isnan(got[[4, 6]]))
    assert np.all(np.abs(got[1:3] - f64(beta)) <= 1e-4 * (1 + np.abs(f64(beta))))       # n is what is left of the mean's rounding, times 1/sqrt(eps)
    for i in (0, 3, 5, 7):
        want = ops.layernorm(x[i:i + 1], None, np.ones(c), f64(beta), 1e-5)[4]
        assert np.all(np.abs(got[i] - want[0]) <= k_of(c) * (np.abs(want[0]) + 1 + 2 * np.abs(f64(beta))))


def test_past_the_caches_and_many_rows():
    """The instances that go past the caches, against the ordinary ones on the same rows (rows are independent: bits are the same)."""
    for c, rows in ((4096, 8192), (256, 131072), (2056, 13000)):
        x = torch.randn((rows, c), device=gu.DEV, dtype=torch.bfloat16)
        gamma, beta = torch.randn(c, device=gu.DEV), torch.randn(c, device=gu.DEV)
        y, mean, rstd = torch.empty_like(x), torch.empty(rows, device=gu.DEV), torch.empty(rows, device=gu.DEV)
        lc.layernorm_fwd(lc.LayerNormDesc(rows, c, dtype=lc.LC_BF16), x, None, gamma, beta, None, y, mean, rstd)
        part, pm, pr = torch.empty((2000, c), dtype=torch.bfloat16, device=gu.DEV), torch.empty(2000, device=gu.DEV), torch.empty(2000, device=gu.DEV)
        lc.layernorm_fwd(lc.LayerNormDesc(2000, c, dtype=lc.LC_BF16), x[-2000:], None, gamma, beta, None, part, pm, pr)
        d, dy = lc.LayerNormDesc(rows, c, dtype=lc.LC_BF16), torch.randn_like(x)
        dx, dg, db = torch.empty_like(x), torch.empty(c, device=gu.DEV), torch.empty(c, device=gu.DEV)
        lc.layernorm_bwd(d, x, dy, None, gamma, mean, rstd, dx, dg, db, gu.workspace(lc.layernorm_bwd_workspace_bytes(d)))
        pd = lc.LayerNormDesc(2000, c, dtype=lc.LC_BF16)
        px = torch.empty_like(part)
        lc.layernorm_bwd(pd, x[-2000:], dy[-2000:], None, gamma, pm, pr, px, torch.empty(c, device=gu.DEV), None, gu.workspace(lc.layernorm_bwd_workspace_bytes(pd)))
        torch.cuda.synchronize()
        assert torch.equal(y[-2000:], part) and torch.equal(mean[-2000:], pm) and torch.equal(rstd[-2000:], pr) and torch.equal(dx[-2000:], px)
        want = dy.double().sum(0)
        assert bool(((db.double() - want).abs() <= (rows + 64) * U * dy.double().abs().sum(0)).all())


def test_a_captured_call_on_another_stream_replays():
    rows, c = 515, 1000
    x, dy = torch.randn((rows, c), device=gu.DEV), torch.randn((rows, c), device=gu.DEV)
    gamma, beta, d = torch.randn(c, device=gu.DEV), torch.randn(c, device=gu.DEV), lc.LayerNormDesc(rows, c)
    ws = gu.workspace(lc.layernorm_bwd_workspace_bytes(d))
    outs = [torch.empty_like(x), torch.empty(rows, device=gu.DEV), torch.empty(rows, device=gu.DEV), torch.empty_like(x), torch.empty(c, device=gu.DEV), torch.empty(c, device=gu.DEV)]

    def call():
        lc.layernorm_fwd(d, x, None, gamma, beta, None, *outs[:3])
        lc.layernorm_bwd(d, x, dy, None, gamma, outs[1], outs[2], outs[3], outs[4], outs[5], ws)

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        call()
    for seed in range(3):
        torch.manual_seed(seed)
        x.copy_(torch.randn((rows, c), device=gu.DEV))
        call()
        torch.cuda.synchronize()
        want = [o.clone() for o in outs]
        for o in outs:
            o.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))


def test_offsets_past_32_bits():
    """1.1 million rows of 4096 bf16, 9 GB each of input and output, with the gradient: the first and last rows against float64, and rows behind the last as they were."""
    rows, c, u8 = 1100000, 4096, 2.0 ** -8
    x = torch.randn((64, c), device=gu.DEV, generator=torch.Generator(gu.DEV).manual_seed(1)).to(torch.bfloat16).repeat((rows + 63) // 64, 1)[:rows]
    y, dx = torch.empty_like(x), torch.empty((rows + 1, c), dtype=torch.bfloat16, device=gu.DEV)
    dx[rows] = 7.0
    gamma, mean, rstd = torch.ones(c, device=gu.DEV), torch.empty(rows, device=gu.DEV), torch.empty(rows, device=gu.DEV)
    d = lc.LayerNormDesc(rows, c, dtype=lc.LC_BF16)
    lc.layernorm_fwd(d, x, None, gamma, None, None, y, mean, rstd)
    dgamma, dbeta = torch.empty(c, device=gu.DEV), torch.empty(c, device=gu.DEV)
    lc.layernorm_bwd(d, x, y, None, gamma, mean, rstd, dx[:rows], dgamma, dbeta, gu.workspace(lc.layernorm_bwd_workspace_bytes(d)))
    for part in (slice(0, 64), slice(rows - 64, rows)):
        v = x[part].double()
        n = (v - v.mean(1, keepdim=True)) / torch.sqrt(v.var(1, unbiased=False, keepdim=True) + 1e-5)
        assert bool(((y[part].double() - n).abs() <= (u8 + 1e-4) * n.abs() + 1e-5).all())
    # rows repeat every 64: so do their gradients, bit for bit
    assert torch.equal(dx[:64], dx[64 * ((rows - 64) // 64):][:64]) and bool((dx[rows] == 7.0).all())
    # dy = y and gamma = 1: dbeta sums y, dgamma y n.  Sums of rows in a fixed order, 1100000 roundings at most of what they have reached
    ys, counts = y[:64].double(), torch.tensor([(rows - i + 63) // 64 for i in range(64)], dtype=torch.float64, device=gu.DEV)[:, None]
    assert bool(((dbeta.double() - (ys * counts).sum(0)).abs() <= rows * 2.0 ** -24 * (ys.abs() * counts).sum(0)).all())
