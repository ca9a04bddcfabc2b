"""Gradients of the layer norm for finite rows whose deviations from their mean leave fp32, and for small ones, against oracle/token_model_ops.py in float64 for the statistics that the forward pass saved.

Tolerances count roundings of u = 2^-24 as everywhere: c/1024 + 64 for a row, rows + 64 for a sum over rows."""
import numpy as np
import pytest
import torch

from oracle import token_model_ops as ops
from paper_1709_05011_amd import larsconv as lc
from paper_1709_05011_amd import synth

import gpu_util as gu

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = {"f32": (lc.LC_F32, torch.float32, 0.0), "bf16": (lc.LC_BF16, torch.bfloat16, 2.0 ** -8)}


def f64(t):
    return t.double().cpu().numpy()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rows,c", [(3, 8), (300, 33), (300, 250), (300, 96), (5, 520), (4, 2049), (3, 8192), (3, 9001), (3, 10240), (2, 20000), (100, 5), (300, 2048)])
@pytest.mark.parametrize("size,eps", [(3.3e38, 0.0), (3.3e38, 1e-5), (1e36, 0.0), (1e-30, 0.0)])
def test_gradients_of_rows_at_the_ends_of_the_range(kind, rows, c, size, eps):
    dtype, t, half = TYPES[kind]
    sign = np.where(synth.uniform01(rows * c, 1).reshape(rows, c) < 0.2, -1.0, 1.0)
    sign[:, 0], sign[:, -1] = -1.0, 1.0
    x = gu.dev((sign * (0.9 + 0.1 * synth.uniform01(rows * c, 2).reshape(rows, c)) * size).astype(np.float32)).to(t)
    gamma, beta = gu.dev(1 + synth.normal((c,), 3, std=0.3)), gu.dev(synth.normal((c,), 4))
    dy = gu.dev(synth.normal((rows, c), 5, std=min(1e20, size))).to(t)       # (gradients that leave something where they are divided by the deviation, and nothing infinite)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    mean, rstd, dg, db = (torch.empty(n, device=gu.DEV) for n in (rows, rows, c, c))
    d = lc.LayerNormDesc(rows, c, eps=eps, dtype=dtype)
    lc.layernorm_fwd(d, x, None, gamma, beta, None, y, mean, rstd)
    lc.layernorm_bwd(d, x, dy, None, gamma, mean, rstd, dx, dg, db, gu.workspace(lc.layernorm_bwd_workspace_bytes(d)))
    torch.cuda.synchronize()
    x64, dy64, m64, r64, g64 = f64(x), f64(dy), f64(mean), f64(rstd), f64(gamma)
    k = (c / 1024 + 64) * U
    _, _, want_rstd, n, want = ops.layernorm(x64, None, g64, f64(beta), float(np.float32(eps)))
    assert np.all(np.abs(f64(y) - want) <= half * (1 + half) * np.abs(want) + k * (1 + half) * (np.abs(n) * np.abs(g64) + np.abs(g64) + np.abs(f64(beta))))
    assert np.all(np.abs(r64 - want_rstd) <= k * want_rstd + 2.0 ** -149)
    want, want_g, want_b = ops.layernorm_bwd(x64, m64, r64, g64, dy64)
    n, a = np.abs((x64 - m64[:, None]) * r64[:, None]), np.abs(dy64 * g64)
    parts = r64[:, None] * (a + np.mean(a, axis=1, keepdims=True) + n * np.mean(a * n, axis=1, keepdims=True))
    assert np.all(np.abs(f64(dx) - want) <= half * (1 + half) * np.abs(want) + k * (1 + half) * parts + 2.0 ** -133)
    assert np.all(np.abs(f64(dg) - want_g) <= (rows + 64) * U * np.sum(np.abs(dy64) * n, axis=0))
    assert np.all(np.abs(f64(db) - want_b) <= (rows + 64) * U * np.sum(np.abs(dy64), axis=0))
