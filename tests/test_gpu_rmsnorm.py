"""GPU parity of the RMS norm (storage type, 8 bits, gradient) against oracle/token_ops.py in float64.

Tolerances count roundings of u = 2^-24 (fp32): a sum of c squares in a block's order takes at most c/1024 + 32 of them, a root, a quotient
and two products 8 more, hence k = c/1024 + 64 relative to the value; a bf16 store adds half a step, 2^-8; an e4m3 code half a step, 2^-4,
or half of its least step, 2^-10 of the scale."""
import numpy as np
import pytest
import torch

from oracle import token_ops as ops
from paper_1709_05011_amd import larsconv as lc
from paper_1709_05011_amd import synth

import gpu_util as gu

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = {"f32": (lc.LC_F32, torch.float32, 0.0), "bf16": (lc.LC_BF16, torch.bfloat16, 2.0 ** -8)}
# one column to rows beyond a block's registers, odd widths, rows beyond the blocks of the backward pass
SHAPES = [(1, 1), (1, 8), (3, 7), (5, 64), (2, 2048), (3, 2049), (4, 4096), (7, 4101), (2, 8192), (2, 8197), (1, 16384), (2, 16385),
          (2, 20001), (1, 40000), (1500, 96), (2100, 33)]


def k_of(c):
    return (c / 1024 + 64) * U


def rows_of(rows, c, seed, dtype, pad=0, offset=0, std=1.0):
    """A device tensor [rows][c] whose rows lie c + pad elements apart, `offset` elements past an aligned address, and its float64 values."""
    whole = torch.full((rows * (c + pad) + offset,), float("nan"), dtype=dtype, device=gu.DEV)
    view = whole[offset:].view(rows, c + pad)[:, :c]
    view.copy_(torch.from_numpy(synth.normal((rows, c), seed, std=std)))
    return view, view.double().cpu().numpy()


def store_of(kind):
    return (lambda v: ops.bf16(v.astype(np.float32))) if kind == "bf16" else (lambda v: v.astype(np.float32).astype(np.float64))


def f64(t):
    return t.double().cpu().numpy()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rows,c", SHAPES)
@pytest.mark.parametrize("residual,pad,offset", [(True, 0, 0), (False, 0, 0), (True, 5, 1), (False, 3, 1)])
def test_forward(kind, rows, c, residual, pad, offset):
    dtype, t, half = TYPES[kind]
    x, x64 = rows_of(rows, c, 1, t, pad, offset)
    r, r64 = rows_of(rows, c, 2, t, 2 * pad, offset, std=3.0) if residual else (None, None)
    gamma = gu.dev(1 + synth.normal((c,), 3, std=0.3))
    total, check_t = gu.guarded((rows, c), t, offset=offset * 4)
    y, check_y = gu.guarded((rows, c), t, offset=offset * 4)
    rstd, check_r = gu.guarded((rows,), torch.float32)
    d = lc.RmsNormDesc(rows, c, x_ld=c + pad, residual_ld=c + 2 * pad, eps=1e-5, dtype=dtype)
    lc.rmsnorm_fwd(d, x, r, gamma, total if residual else None, y, rstd)
    torch.cuda.synchronize()
    h, want_rstd, want = ops.rmsnorm(x64, r64, f64(gamma), float(np.float32(1e-5)), store_of(kind))
    for check in (check_t, check_y, check_r):
        check()
    if residual:
        assert np.array_equal(f64(total), h)
    assert np.all(np.abs(f64(rstd) - want_rstd) <= k_of(c) * want_rstd)
    assert np.all(np.abs(f64(y) - want) <= (half * (1 + half) + k_of(c)) * np.abs(want))


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rows,c", SHAPES)
@pytest.mark.parametrize("group", [0, 32, 128, 512])
def test_forward_in_8_bits(kind, rows, c, group):
    dtype, t, _ = TYPES[kind]
    pad = c % 3
    x, x64 = rows_of(rows, c, 4, t, pad)
    r, r64 = rows_of(rows, c, 5, t)
    gamma = gu.dev(1 + synth.normal((c,), 6, std=0.3))
    groups = -(-c // group) if group else 1
    y, check_y = gu.guarded((rows, c), torch.float8_e4m3fn)
    s, check_s = gu.guarded((rows, groups), torch.float32)
    lc.rmsnorm_fwd_q8(lc.RmsNormDesc(rows, c, x_ld=c + pad, dtype=dtype), x, r, gamma, None, y, s, group)
    torch.cuda.synchronize()
    check_y()
    check_s()
    want = ops.rmsnorm(x64, r64, f64(gamma), float(np.float32(1e-5)), store_of(kind))[2]
    want_s = ops.quantise_rows(want, group)[1]
    got_s, got = f64(s), y.float().double().cpu().numpy()
    assert np.all(np.abs(got_s - want_s) <= k_of(c) * want_s)
    wide = np.repeat(got_s, group or c, axis=1)[:, :c]
    assert np.all(np.abs(got * wide - want) <= np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** -10 * wide) + k_of(c) * np.abs(want))
    top = np.maximum.reduceat(np.abs(got), np.arange(0, c, group or c), axis=1)
    assert np.array_equal(top, np.where(got_s > 2.0 ** -126, 448.0, 0.0))     # the largest of a group takes the largest code; zeros stay zeros


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rows,c", SHAPES)
@pytest.mark.parametrize("joined,pad", [(True, 0), (False, 3)])
def test_backward(kind, rows, c, joined, pad):
    dtype, t, half = TYPES[kind]
    h, h64 = rows_of(rows, c, 7, t, pad, std=2.0)
    dy, dy64 = rows_of(rows, c, 8, t, 0, pad, std=0.1)
    dt, dt64 = rows_of(rows, c, 9, t, 0, pad, std=0.1) if joined else (None, None)
    gamma = gu.dev(1 + synth.normal((c,), 10, std=0.3))
    rstd64 = 1 / np.sqrt(np.mean(h64 ** 2, axis=1) + 1e-5)
    rstd = gu.dev(rstd64.astype(np.float32))
    rstd64 = f64(rstd)
    dx, check_x = gu.guarded((rows, c), t)
    dg, check_g = gu.guarded((c,), torch.float32)
    d = lc.RmsNormDesc(rows, c, dtype=dtype)
    ws = gu.workspace(lc.rmsnorm_bwd_workspace_bytes(d))
    lc.rmsnorm_bwd(d, h, dy, dt, gamma, rstd, dx, dg, ws, h_ld=c + pad)
    torch.cuda.synchronize()
    check_x()
    check_g()
    g64 = f64(gamma)
    want, want_g = ops.rmsnorm_bwd(h64, rstd64, g64, dy64, dt64)
    n, a = np.abs(h64 * rstd64[:, None]), np.abs(dy64 * g64)
    parts = rstd64[:, None] * (a + n * np.mean(a * n, axis=1, keepdims=True)) + (0 if dt is None else np.abs(dt64))
    assert np.all(np.abs(f64(dx) - want) <= half * (1 + half) * np.abs(want) + (k_of(c) * (1 + half)) * parts)
    assert np.all(np.abs(f64(dg) - want_g) <= (rows + 64) * U * np.sum(np.abs(dy64) * n, axis=0))


def test_the_gradient_against_differences():
    """Central differences of the float64 sum of y * dy through the kernel's own forward pass, fp32: a step of 2^-6 keeps its rounding under 1e-3."""
    rows, c, e = 2, 24, 2.0 ** -6
    x = synth.normal((rows, c), 11)
    dy, gamma = synth.normal((rows, c), 12), gu.dev(1 + synth.normal((c,), 13, std=0.3))
    d = lc.RmsNormDesc(rows, c, eps=1e-3)
    y, rstd = torch.empty((rows, c), device=gu.DEV), torch.empty(rows, device=gu.DEV)

    def forward(a):
        lc.rmsnorm_fwd(d, gu.dev(a.astype(np.float32)), None, gamma, None, y, rstd)
        return float(np.sum(f64(y) * dy))

    forward(x)
    dx, dg, ws = torch.empty((rows, c), device=gu.DEV), torch.empty(c, device=gu.DEV), gu.workspace(lc.rmsnorm_bwd_workspace_bytes(d))
    lc.rmsnorm_bwd(d, gu.dev(x), gu.dev(dy), None, gamma, rstd, dx, dg, ws)
    got = f64(dx)
    for i, j in [(0, 0), (0, 23), (1, 5), (1, 12)]:
        up, down = x.copy(), x.copy()
        up[i, j] += np.float32(e)
        down[i, j] -= np.float32(e)
        numeric = (forward(up) - forward(down)) / float(up[i, j].astype(np.float64) - down[i, j].astype(np.float64))
        assert abs(numeric - got[i, j]) < 2e-3 * max(1.0, abs(got[i, j]))


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("c", [96, 5000, 17000])
def test_total_in_the_residuals_own_buffer(kind, c):
    dtype, t, _ = TYPES[kind]
    x, _ = rows_of(3, c, 14, t)
    r, _ = rows_of(3, c, 15, t)
    gamma, d = gu.dev(1 + synth.normal((c,), 16, std=0.3)), lc.RmsNormDesc(3, c, dtype=dtype)
    y0, y1, total = (torch.empty((3, c), dtype=t, device=gu.DEV) for _ in range(3))
    lc.rmsnorm_fwd(d, x, r, gamma, total, y0)
    lc.rmsnorm_fwd(d, x, r, gamma, r, y1)
    torch.cuda.synchronize()
    assert torch.equal(total, r) and torch.equal(y0, y1)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("c", [130, 3000, 17000])
def test_rows_of_zeros_infinities_and_nan(kind, c):
    """A row of zeros gives zeros (and the least scale); an infinity or a NaN stays in its own row."""
    dtype, t, _ = TYPES[kind]
    x, _ = rows_of(5, c, 17, t)
    x[1] = 0
    x[2, c // 2] = float("nan")
    x[3, 0] = float("inf")
    gamma, d = gu.dev(1 + synth.normal((c,), 18, std=0.3)), lc.RmsNormDesc(5, c, dtype=dtype)
    y, y8, s = torch.empty((5, c), dtype=t, device=gu.DEV), torch.empty((5, c), dtype=torch.float8_e4m3fn, device=gu.DEV), torch.empty(5, device=gu.DEV)
    lc.rmsnorm_fwd(d, x, None, gamma, None, y)
    lc.rmsnorm_fwd_q8(d, x, None, gamma, None, y8, s)
    torch.cuda.synchronize()
    assert not y[1].any() and float(s[1]) == 2.0 ** -126 and not y8[1].float().any()
    assert y[2].isnan().all() and y8[2].float().isnan().all()
    assert y[3, 0].isnan() and not y[3, 1:].any() and y8[3, 0].float().isnan() and not y8[3, 1:].float().any()
    assert y[[0, 4]].isfinite().all() and y8[[0, 4]].float().isfinite().all()


def test_no_rows_gives_a_zero_gradient_of_gamma():
    dg = torch.full((77,), 3.0, device=gu.DEV)
    lc.rmsnorm_bwd(lc.RmsNormDesc(0, 77), None, None, None, None, None, None, dg)
    torch.cuda.synchronize()
    assert not dg.any()


def test_another_stream_and_bit_identical_reruns():
    rows, c = 700, 1000
    h, _ = rows_of(rows, c, 19, torch.bfloat16)
    dy, _ = rows_of(rows, c, 20, torch.bfloat16)
    gamma, d = gu.dev(1 + synth.normal((c,), 21, std=0.3)), lc.RmsNormDesc(rows, c, dtype=lc.LC_BF16)
    ws, got = gu.workspace(lc.rmsnorm_bwd_workspace_bytes(d)), []
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for stream in (torch.cuda.current_stream(), side):
        y, rstd, dx, dg = torch.empty_like(h), torch.empty(rows, device=gu.DEV), torch.empty_like(h), torch.empty(c, device=gu.DEV)
        torch.cuda.synchronize()
        lc.rmsnorm_fwd(d, h, None, gamma, None, y, rstd, stream=stream)
        lc.rmsnorm_bwd(d, h, dy, None, gamma, rstd, dx, dg, ws, stream=stream)
        torch.cuda.synchronize()
        got.append((y, rstd, dx, dg))
    assert all(torch.equal(a, b) for a, b in zip(*got))


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("c", [96, 2048, 17000])
@pytest.mark.parametrize("group", [0, 32])
@pytest.mark.parametrize("up,gain", [(50, 90), (-50, -80)])
def test_powers_of_two_move_the_scales_and_not_the_codes(kind, c, group, up, gain):
    """Every step scales exactly by powers of two without eps, also where total * gamma itself (2^140, 2^-130) is out of fp32's range."""
    dtype, t, _ = TYPES[kind]
    x, _ = rows_of(3, c, 19, t)
    gamma = gu.dev(1 + synth.normal((c,), 20, std=0.3))
    groups = -(-c // group) if group else 1
    out = []
    for a, b in [(0, 0), (up, gain)]:
        y, s = torch.empty((3, c), dtype=torch.float8_e4m3fn, device=gu.DEV), torch.empty((3, groups), device=gu.DEV)
        lc.rmsnorm_fwd_q8(lc.RmsNormDesc(3, c, eps=0.0, dtype=dtype), x * 2.0 ** a, None, gamma * 2.0 ** b, None, y, s, group)
        torch.cuda.synchronize()
        out.append((y.view(torch.uint8), s))
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1] * 2.0 ** gain, out[1][1])


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rows,c", [(1, 16), (33, 64), (70, 72), (17, 128), (700, 128), (9, 129), (301, 200), (500, 256), (5000, 64), (40000, 40)])
def test_narrow_rows(kind, rows, c):
    """Several rows of a wave: blocks that end within their rows, rows that end within a lane's columns, groups as wide as a row and wider."""
    for residual, pad, offset in [(True, 0, 0), (False, 5, 1)]:
        test_forward(kind, rows, c, residual, pad, offset)
    for group in (0, 32, 512):
        test_forward_in_8_bits(kind, rows, c, group)
    for joined, pad in [(True, 0), (False, 3)]:
        test_backward(kind, rows, c, joined, pad)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rows,c", [(3, 130), (300, 130), (3, 3000), (3, 17000)])
@pytest.mark.parametrize("group", [0, 128])
def test_an_infinite_factor_stays_in_its_group(kind, rows, c, group):
    """The group's scale is infinite: the column itself has no number for a code, its neighbours' quotient is 0, other groups are as without it."""
    dtype, t, _ = TYPES[kind]
    x, _ = rows_of(rows, c, 21, t)
    gamma = gu.dev(1 + synth.normal((c,), 22, std=0.3))
    groups = -(-c // group) if group else 1
    out = []
    for _ in range(2):
        y, s = torch.empty((rows, c), dtype=torch.float8_e4m3fn, device=gu.DEV), torch.empty((rows, groups), device=gu.DEV)
        lc.rmsnorm_fwd_q8(lc.RmsNormDesc(rows, c, dtype=dtype), x, None, gamma, None, y, s, group)
        torch.cuda.synchronize()
        out.append((y.float(), s))
        gamma[5] = float("inf")
    (y0, s0), (y1, s1) = out
    end = group or c
    assert torch.all(s1[:, 0].isinf()) and torch.all(y1[:, 5].isnan())
    assert not y1[:, :5].any() and not y1[:, 6:end].any()
    assert torch.equal(y1[:, end:], y0[:, end:]) and torch.equal(s1[:, 1:], s0[:, 1:])


def test_gradient_of_more_columns_than_a_launch_has_threads_for():
    """dgamma's sum takes 1024 threads for 64 columns: 2^32 of them from 2^28 columns on.  One row in three, so that a wrong tile of columns shows."""
    rows, c = 3, (1 << 28) + 37
    gen = torch.Generator(device=gu.DEV).manual_seed(3)
    h, dy = (torch.randn((rows, c), generator=gen, device=gu.DEV, dtype=torch.bfloat16) for _ in range(2))
    gamma, dx, dg = torch.ones(c, device=gu.DEV), torch.empty_like(h), torch.full((c,), float("nan"), device=gu.DEV)
    rstd = torch.tensor([1.0, 0.5, 2.0], device=gu.DEV)
    d = lc.RmsNormDesc(rows, c, dtype=lc.LC_BF16)
    lc.rmsnorm_bwd(d, h, dy, None, gamma, rstd, dx, dg, gu.workspace(lc.rmsnorm_bwd_workspace_bytes(d)))
    torch.cuda.synchronize()
    for at in range(0, c, 1 << 26):                  # rstd a power of two and products of two bf16 values: three exact terms, two roundings
        terms = h[:, at:at + (1 << 26)].float() * rstd[:, None] * dy[:, at:at + (1 << 26)].float()
        off = (dg[at:at + (1 << 26)] - terms.double().sum(0)).abs()
        assert bool((off <= 3 * U * terms.abs().double().sum(0)).all()), at


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rows,c", [(9, 1), (9, 24), (700, 100), (9, 512), (9, 5000), (9, 8200), (9, 16384), (9, 17000), (9, 9001)])
@pytest.mark.parametrize("eps", [0.0, 1e-40, 1e-33, 1e-5])
def test_rows_whose_squares_leave_fp32(kind, rows, c, eps):
    """Ordinary rows beside rows of 1e-36 to 1e37: sums of squares under the normal range or beyond the largest number, with an eps that hides the small ones and with one that
    does not.  The result is the definition's; the tolerances are those of the forward pass, and eight more roundings of an rstd under 2^-126 (which holds 2^-149 or 2^-21 of
    1e-37's neighbours)."""
    dtype, t, half = TYPES[kind]
    sizes = np.array([1.0, 1e-36, 1e-25, 1e-20, 1e-19, 1e18, 1e19, 1e30, 2e37])
    x = synth.normal((rows, c), 23).astype(np.float64) * sizes[np.arange(rows) % 9][:, None]
    x = torch.from_numpy(x).to(t).to(gu.DEV)
    gamma, d = gu.dev(1 + synth.normal((c,), 24, std=0.3)), lc.RmsNormDesc(rows, c, eps=eps, dtype=dtype)
    y, rstd = torch.empty((rows, c), dtype=t, device=gu.DEV), torch.empty(rows, device=gu.DEV)
    y8, s = torch.empty((rows, c), dtype=torch.float8_e4m3fn, device=gu.DEV), torch.empty((rows, -(-c // 32)), device=gu.DEV)
    lc.rmsnorm_fwd(d, x, None, gamma, None, y, rstd)
    lc.rmsnorm_fwd_q8(d, x, None, gamma, None, y8, s, 32)
    torch.cuda.synchronize()
    _, want_rstd, want = ops.rmsnorm(f64(x), None, f64(gamma), float(np.float32(eps)))
    small = 8 * U * (want_rstd < 2.0 ** -120)[:, None]
    assert np.all(np.abs(f64(rstd) - want_rstd) <= (k_of(c) + small[:, 0]) * want_rstd)
    low = 2.0 ** -130                                  # (an eps beside rows of 1e-36 takes their y under the normal range)
    assert np.all(np.abs(f64(y) - want) <= (half * (1 + half) + k_of(c) + small) * np.abs(want) + low)
    want_s = ops.quantise_rows(want, 32)[1]
    assert np.all(np.abs(f64(s) - want_s) <= k_of(c) * want_s)
    wide = np.repeat(f64(s), 32, axis=1)[:, :c]
    got = y8.float().double().cpu().numpy() * wide
    assert np.all(np.abs(got - want) <= np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** -10 * wide) + k_of(c) * np.abs(want))
