"""What the header says of the Newton-Schulz steps' results: where singular values come to, and how far results are off beside those of fp32 products."""
import numpy as np
import pytest
import torch

from oracle import token_model_ops as ops
from paper_1709_05011_amd import larsconv as lc

import gpu_util as gu
from test_gpu_newton_schulz import matrix, on_the_device

pytestmark = pytest.mark.gpu


def test_where_singular_values_come_to():
    """Five steps: what is 0.007 of the norm or more comes to between 0.68 and 1.14, what is 0.002 or more to between 0.68 and 1.21, and less grows by 3.4445 a step at most.  Values of a diagonal matrix
    go through the steps by themselves; between products they are stored 15 times with 2^-22, which the polynomial's slope multiplies by up to 3.4445 a step."""
    s = np.exp(np.linspace(np.log(1e-5), np.log(0.5), 120))
    x = np.zeros((120, 130), np.float32)
    x[np.arange(120), np.arange(120)[::-1]] = s
    x[0, 119] = 0.4
    x64 = x.astype(np.float64)
    d, y = lc.NewtonSchulzDesc(1, 120, 130), torch.empty((120, 130), device=gu.DEV)
    lc.newton_schulz(d, gu.dev(x), y, gu.workspace(lc.newton_schulz_workspace_bytes(d)))
    part = (x64.max(axis=1) / (np.sqrt(np.sum(x64 ** 2)) + 1e-7))
    got, off = y.double().cpu().numpy().max(axis=1), 15 * 3.4445 ** 5 * 2.0 ** -22
    assert np.all(np.abs(got - ops.newton_schulz(x64).max(axis=1)) <= off)
    assert got[part >= 0.007].min() >= 0.68 - off and got[part >= 0.007].max() <= 1.14 + off
    assert got[part >= 0.002].min() >= 0.68 - off and got[part >= 0.002].max() <= 1.21 + off
    assert got[(part >= 0.002) & (part < 0.007)].max() > 1.15      # (the larger bound is met)
    assert np.all(got[part < 0.002] <= 3.4445 ** 5 * part[part < 0.002] + off)


@pytest.mark.parametrize("how", ["normal", "gradient", "low rank"])
@pytest.mark.parametrize("rows,cols", [(4, 4), (8, 8), (16, 2000), (2000, 16), (48, 48), (64, 256), (64, 2304), (100, 2000), (128, 1152)])
def test_matrices_with_a_short_side_beside_fp32_products(rows, cols, how):
    """A value rounded to a pair is off by up to 2^-22, four times fp32's 2^-24, and sums are fp32 on either side: on the average of sixteen matrices errors are at most four times those of fp32 products."""
    off, plain = [], []
    for seed in range(16):
        x = gu.dev(matrix(rows, cols, 10 * seed + 7, how))
        y, d = torch.empty_like(x), lc.NewtonSchulzDesc(1, rows, cols)
        lc.newton_schulz(d, x, y, gu.workspace(lc.newton_schulz_workspace_bytes(d)))
        want = on_the_device(x, torch.float64)
        error = lambda v: float((v.double() - want).norm() / want.norm())
        off.append(error(y))
        plain.append(error(on_the_device(x, torch.float32)))
    assert np.mean(off) <= 4 * np.mean(plain), (np.mean(off), np.mean(plain))
