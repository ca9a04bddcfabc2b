"""The layer norm's gradients where a thread of the backward pass walks more than one row, against oracle/token_model_ops.py in float64: blocks with a row at a time, several rows of a wave, rows that go
by in passes (whose shares are ranges of rows), and the instances past the caches.

Tolerances count roundings of u = 2^-24: dx as a row's (c/1024 + 64 of them); dgamma and dbeta have sums of rows / 64 at most in a thread (there are 64 shares or more, or one
a row), of a wave and a block behind it (8), of up to 4096 shares in 16 groups by eights (32, 3 and 16), and products of four roundings: rows / 64 + 80.  A share lost would be 1/64 of the sum or more than a row's product."""
import numpy as np
import pytest
import torch

from oracle import token_model_ops as ops
from paper_1709_05011_amd import larsconv as lc

import gpu_util as gu

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = {"f32": (lc.LC_F32, torch.float32, 0.0), "bf16": (lc.LC_BF16, torch.bfloat16, 2.0 ** -8)}
# blocks of whole rows (256 to 4096 waves of them), rows of 8, 16 and 32 lanes, rows that go by in passes (of fp32 also odd ones over 8192 columns); fp32 from 96 MB on has no other instances, bf16 has
SHAPES = [(515, 1000), (515, 1537), (3000, 264), (3000, 2049), (1030, 4096), (5000, 520), (700, 8200), (600, 10240), (300, 16384), (40000, 48), (33001, 64), (20000, 100), (10001, 250), (70000, 256),
          (200, 7), (70000, 1), (130, 17000), (130, 9001), (6000, 3001), (9000, 2048), (300000, 63)]


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rows,c", SHAPES)
@pytest.mark.parametrize("joined,shift", [(False, True), (True, False)])
def test_gradients_of_many_rows(kind, rows, c, joined, shift):
    dtype, t, half = TYPES[kind]
    gen = torch.Generator(gu.DEV).manual_seed(rows + c)
    normal = lambda *shape: torch.randn(shape, device=gu.DEV, generator=gen)
    h, dy = (normal(rows, c) * 2 + 0.7).to(t), (normal(rows, c) * 0.1 + 0.02).to(t)
    dt = (normal(rows, c) * 0.1).to(t) if joined else None
    gamma = 1 + 0.3 * normal(c)
    h64, dy64, g64 = h.double(), dy.double(), gamma.double()
    mean, rstd = h64.mean(1).float(), (1 / torch.sqrt(h64.var(1, unbiased=False) + 1e-5)).float()
    dx, check_x = gu.guarded((rows, c), t)
    dg, check_g = gu.guarded((c,), torch.float32)
    db, check_b = gu.guarded((c,), torch.float32)
    d = lc.LayerNormDesc(rows, c, dtype=dtype)
    ws = gu.workspace(lc.layernorm_bwd_workspace_bytes(d))
    ws.fill_(0xff)
    lc.layernorm_bwd(d, h, dy, dt, gamma, mean, rstd, dx, dg, db if shift else None, ws)
    torch.cuda.synchronize()
    for check in (check_x, check_g, check_b):
        check()
    cpu = lambda v: v.double().cpu().numpy()
    want, want_g, want_b = ops.layernorm_bwd(cpu(h), cpu(mean), cpu(rstd), cpu(gamma), cpu(dy), None if dt is None else cpu(dt))
    n, a = torch.abs((h64 - mean.double()[:, None]) * rstd.double()[:, None]), torch.abs(dy64 * g64)
    parts = rstd.double()[:, None] * (a + a.mean(1, keepdim=True) + n * (a * n).mean(1, keepdim=True)) + (0 if dt is None else dt.double().abs())
    k = (c / 1024 + 64) * U
    assert np.all(np.abs(cpu(dx) - want) <= half * (1 + half) * np.abs(want) + k * (1 + half) * cpu(parts))
    assert np.all(np.abs(cpu(dg) - want_g) <= (rows / 64 + 80) * U * cpu((dy64.abs() * n).sum(0)))
    if shift:
        assert np.all(np.abs(cpu(db) - want_b) <= (rows / 64 + 80) * U * cpu(dy64.abs().sum(0)))
    else:
        assert bool(torch.isnan(db).all())


def test_gradients_of_scale_and_shift_past_32_bits():
    """1.1 million rows of 4096 bf16 whose rows repeat every 64: dgamma and dbeta are the sums of 64 rows' shares, each as often as its row occurs."""
    rows, c = 1100000, 4096
    x = torch.randn((64, c), device=gu.DEV, generator=torch.Generator(gu.DEV).manual_seed(1)).to(torch.bfloat16)
    dy = torch.randn((64, c), device=gu.DEV, generator=torch.Generator(gu.DEV).manual_seed(2)).to(torch.bfloat16)
    mean, rstd = x.double().mean(1).float(), (1 / torch.sqrt(x.double().var(1, unbiased=False) + 1e-5)).float()
    times = (rows + 63) // 64
    every = lambda v: v.repeat(*([times] + [1] * (v.dim() - 1)))[:rows]
    dx, dg, db = torch.empty((rows, c), dtype=torch.bfloat16, device=gu.DEV), torch.empty(c, device=gu.DEV), torch.empty(c, device=gu.DEV)
    d = lc.LayerNormDesc(rows, c, dtype=lc.LC_BF16)
    lc.layernorm_bwd(d, every(x), every(dy), None, torch.ones(c, device=gu.DEV), every(mean), every(rstd), dx, dg, db, gu.workspace(lc.layernorm_bwd_workspace_bytes(d)))
    n = (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
    counts = torch.tensor([(rows - i + 63) // 64 for i in range(64)], dtype=torch.float64, device=gu.DEV)[:, None]
    # a block adds rows / 512 products of four roundings, the 512 shares are added by eights in 16 groups
    steps = rows // 512 + 64
    for got, share in ((dg, dy.double() * n), (db, dy.double())):
        assert bool(((got.double() - (share * counts).sum(0)).abs() <= steps * U * (share.abs() * counts).sum(0)).all())
