"""Pins of the float64 definitions in oracle/token_ops.py: hand-worked values, other people's casts (torch), finite differences."""
import numpy as np
import pytest
import torch

from oracle import token_ops as ops


def test_e4m3_and_bf16_are_the_formats_torch_knows():
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy()
    values = np.unique(codes[np.isfinite(codes)])
    assert values.max() == 448.0
    assert np.array_equal(ops.e4m3(values), values)
    x = np.concatenate([(values[1:] + values[:-1]) / 2, values * 1.0301, np.float32([1e-4, 3e-3, 447.9])]).astype(np.float32)
    x = x[np.abs(x) <= 448]
    assert np.array_equal(ops.e4m3(x), torch.from_numpy(x).to(torch.float8_e4m3fn).double().numpy())
    y = np.random.default_rng(0).normal(size=1000).astype(np.float32)
    assert np.array_equal(ops.bf16(y), torch.from_numpy(y).bfloat16().double().numpy())


def test_rmsnorm_by_hand():
    h, rstd, y = ops.rmsnorm(np.array([[1.0, 2.0]]), np.array([[2.0, 2.0]]), np.array([1.0, 10.0]), 0.0)
    assert np.array_equal(h, [[3.0, 4.0]])
    assert np.allclose(rstd, 1 / np.sqrt(12.5)) and np.allclose(y, [[3 / np.sqrt(12.5), 40 / np.sqrt(12.5)]])
    q, s = ops.quantise_rows(np.array([[1.0, -3.5, 0.01, 0.0]]), 2)
    assert np.allclose(s, [[3.5 / 448, 0.01 / 448]]) and np.array_equal(q, [[128.0, -448.0, 448.0, 0.0]])
    assert np.array_equal(ops.quantise_rows(np.zeros((1, 3)), 0)[1], [[2.0 ** -126]])


def test_rmsnorm_gradient_against_differences_and_autograd():
    rng = np.random.default_rng(1)
    x, r, g, dy, dt = rng.normal(size=(3, 7)), rng.normal(size=(3, 7)), rng.normal(size=7), rng.normal(size=(3, 7)), rng.normal(size=(3, 7))
    f = lambda x, g: float(np.sum(ops.rmsnorm(x, r, g, 1e-3)[2] * dy) + np.sum((x + r) * dt))
    h, rstd, _ = ops.rmsnorm(x, r, g, 1e-3)
    dx, dg = ops.rmsnorm_bwd(h, rstd, g, dy, dt)
    e = 1e-6
    for i in range(3):
        for j in range(7):
            d = np.zeros_like(x)
            d[i, j] = e
            assert abs((f(x + d, g) - f(x - d, g)) / (2 * e) - dx[i, j]) < 1e-7
    for j in range(7):
        d = np.zeros_like(g)
        d[j] = e
        assert abs((f(x, g + d) - f(x, g - d)) / (2 * e) - dg[j]) < 1e-7
    tx, tg = torch.tensor(x, requires_grad=True), torch.tensor(g, requires_grad=True)
    th = tx + torch.tensor(r)
    ty = th * torch.rsqrt((th * th).mean(1, keepdim=True) + 1e-3) * tg
    ((ty * torch.tensor(dy)).sum() + (th * torch.tensor(dt)).sum()).backward()
    assert np.allclose(tx.grad.numpy(), dx, atol=1e-12) and np.allclose(tg.grad.numpy(), dg, atol=1e-12)


def test_token_logprob_by_hand():
    z = np.log(np.array([[1.0, 2.0, 4.0, 1.0]]))
    lp, ent, lse, ids, top = ops.token_logprob(z, np.array([2]), 3)
    p = np.array([1, 2, 4, 1]) / 8
    assert np.allclose(lp, np.log(0.5)) and np.allclose(lse, np.log(8)) and np.allclose(ent, -np.sum(p * np.log(p)))
    assert np.array_equal(ids, [[2, 1, 0]]) and np.allclose(top, np.log(p[[2, 1, 0]]))
    lp, ent, lse, ids, top = ops.token_logprob(np.array([[0.0, -np.inf], [-np.inf, -np.inf]]), np.array([1, -1]), 2)
    assert lp[0] == -np.inf and ent[0] == 0 and lse[0] == 0 and np.array_equal(ids, [[0, -1], [-1, -1]])
    assert lp[1] == 0 and ent[1] == 0 and lse[1] == -np.inf
    assert not ops.token_logprob_bwd(np.array([[-np.inf] * 2]), np.array([0]), np.ones(1), np.ones(1)).any()


def test_token_logprob_gradient_against_differences_and_autograd():
    rng = np.random.default_rng(2)
    z, t, a, b = rng.normal(size=(4, 9)), np.array([0, 8, -1, 9]), rng.normal(size=4), rng.normal(size=4)
    f = lambda z: float(np.dot(a, ops.token_logprob(z, t)[0]) + np.dot(b, ops.token_logprob(z, t)[1]))
    dz, e = ops.token_logprob_bwd(z, t, a, b), 1e-6
    for i in range(4):
        for j in range(9):
            d = np.zeros_like(z)
            d[i, j] = e
            assert abs((f(z + d) - f(z - d)) / (2 * e) - dz[i, j]) < 1e-8
    tz = torch.tensor(z, requires_grad=True)
    logp = torch.log_softmax(tz, 1)
    loss = a[0] * logp[0, 0] + a[1] * logp[1, 8] - (torch.tensor(b) * (logp.exp() * logp).sum(1)).sum()
    loss.backward()
    assert np.allclose(tz.grad.numpy(), dz, atol=1e-12)


def test_adamw_against_torchs_own():
    rng = np.random.default_rng(3)
    w, g = rng.normal(size=20), rng.normal(size=(3, 20))
    p = torch.tensor(w, requires_grad=True)
    opt = torch.optim.AdamW([p], lr=0.02, betas=(0.8, 0.95), eps=1e-6, weight_decay=0.1)
    m = v = np.zeros(20)
    for t in range(3):
        p.grad = torch.tensor(g[t])
        opt.step()
        w, m, v = ops.adamw(w, g[t], m, v, 0.02, 0.8, 0.95, 1e-6, 0.1, t + 1)
    assert np.allclose(w, p.detach().numpy(), rtol=1e-12, atol=1e-14)
    by_32, v_32 = ops.adam_states_as_rounded(g[0], m, v, 0.8, 0.95, 0.5)
    _, m, v = ops.adamw(w, g[0], np.float32(m), np.float32(v), 0, 0.8, 0.95, 1e-6, 0, 4, 0.5)
    assert by_32.dtype == np.float32 and np.allclose(by_32, m, rtol=1e-6, atol=1e-7) and np.allclose(v_32, v, rtol=1e-6)


def test_power_scales():
    for amax, most, want in [(0.0, 448.0, 1.0), (448.0, 448.0, 1.0), (449.0, 448.0, 2.0), (224.0, 448.0, 0.5), (1.0, 448.0, 2.0 ** -8), (1e-300, 448.0, 2.0 ** -126),
                             (57344.0 * 8, 57344.0, 8.0)]:
        assert ops.power_scale(amax, most) == want


def test_dithered_e5m2():
    values = torch.arange(124, dtype=torch.uint8).view(torch.float8_e5m2).double().numpy()      # 0 .. 57344
    assert np.array_equal(ops.e5m2_dithered(values, 0), values)                   # on the grid nothing moves, whatever the bits
    assert np.array_equal(ops.e5m2_dithered(values, 2.0 ** 21 - 1), values)
    assert ops.e5m2_dithered(np.array([1e-30]), 0)[0] == 2.0 ** -16               # above zero stays above zero
    x = 1.25 + 0.25 * 0.3                                                          # between 1.25 and 1.5
    bits = ops.dither21(np.arange(20000), 7)
    assert bits.min() >= 0 and bits.max() < 2 ** 21
    got = ops.e5m2_dithered(np.full(20000, x), bits)
    assert set(np.unique(got)) == {1.25, 1.5} and abs(np.mean(got) - x) < 5 * 0.25 * np.sqrt(0.3 * 0.7 / 20000)


def test_dither_is_even_and_differs_by_seed():
    a, b = ops.dither21(np.arange(30000), 1), ops.dither21(np.arange(30000), 2)
    for bits in (a, b, (a + b) % 2 ** 21, (a[1:] - a[:-1]) % 2 ** 21, (a - b) % 2 ** 21):
        count = np.bincount((bits // 2 ** 17).astype(int), minlength=16)
        expected = bits.size / 16
        assert np.sum((count - expected) ** 2 / expected) < 60                     # chi-square of 15 degrees: mean 15, P(> 60) below 1e-6
