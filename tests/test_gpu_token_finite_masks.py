"""Token log probabilities where finite numbers far from zero stand for masks, or are a row's largest: the product of such a logit with log2 e is off by more than
exponents can carry (half a unit of 1.4e10 is 512), a whole lane's, wave's or row's values at a time.  Against oracle/token_ops.py in float64; the tolerances are those of
test_gpu_token_logprob.py, whose counts do not depend on where the logits lie: distances from the maximum are rounded once, and lse once to its own size."""
import numpy as np
import pytest
import torch

from oracle import token_ops as ops
from paper_1709_05011_amd import larsconv as lc
from paper_1709_05011_amd import synth

import gpu_util as gu
from test_gpu_token_logprob import TYPES, U, check_forward, f64, run, tol, tokens_of

pytestmark = pytest.mark.gpu


def in_range(a):
    """Differences of the largest and the lowest that fp32 does not hold are infinities of their sign."""
    return np.where(np.abs(a) > np.finfo(np.float32).max, np.copysign(np.inf, a), a)


def check(kind, z, t64, top):
    """Forward with and without alternatives, and the gradient, of the rows z (a device tensor)."""
    dtype, _, half = TYPES[kind]
    rows, vocab = z.shape
    z64, tokens = f64(z), gu.dev(t64.astype(np.int32))
    place = np.arange(vocab)
    for n in {0, top}:
        got = run(dtype, z, tokens, vocab, n)
        check_forward(vocab, got, [in_range(a) for a in ops.token_logprob(z64, t64, n)], n)
    d, (lp, ent, lse), _, _ = got
    one, dz = torch.ones(rows, device=gu.DEV), torch.empty_like(z)
    lc.token_logprob_bwd(d, z, tokens, lse, ent, one, 0.5 * one, dz)
    torch.cuda.synchronize()
    m = np.max(z64, axis=1, keepdims=True)
    m = np.where(m == -np.inf, 0.0, m)
    with np.errstate(divide="ignore"):
        logp = (z64 - m) - np.log(np.sum(np.exp(z64 - m), axis=1, keepdims=True))
    empty = np.all(z64 == -np.inf, axis=1, keepdims=True)
    logp = np.where(empty, -np.inf, logp)
    e64 = ops.token_logprob(z64, t64, 0)[1][:, None]
    p, fine = np.exp(logp), np.where(np.exp(logp) > 0, logp, 0.0)
    counts = ((t64 >= 0) & (t64 < vocab))[:, None] & ~empty
    want = counts * ((place == t64[:, None]) - p) - 0.5 * p * (fine + e64)
    # p by exp(d - log S), and half a unit of lse where it is formed from lse (|lse| at most 256 in fp32, 16384 in bf16)
    rel = tol(vocab) * (2 + e64) + U * (4 * np.abs(fine) + (16384 if kind == "bf16" else 256))
    bound = p * (1.5 + np.abs(fine) + e64) * rel + 2 * U
    assert np.all(np.abs(f64(dz) - want) <= half * (1 + half) * np.abs(want) + (1 + half) * bound)


def stretches(vocab):
    """A thread's eight columns, its sixteen, a wave's round of them, three rounds and a bit: where they fit."""
    return [(a, b) for a, b in [(0, 8), (16, 32), (512, 1536), (vocab // 2 // 1024 * 1024, vocab // 2 // 1024 * 1024 + 3100), (8, vocab - 9)] if a < b <= vocab]


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [40, 700, 9001, 40000])
@pytest.mark.parametrize("mask", [-1e6, -1e7, -1e9, -1e10, -1e20, -1e30, -2.2e38, -2.4e38])
def test_stretches_of_a_finite_mask_in_ordinary_rows(kind, vocab, mask):
    t = TYPES[kind][1]
    parts = stretches(vocab)
    z = synth.normal((len(parts) + 2, vocab), 31, std=3.0)
    for row, (a, b) in enumerate(parts):
        z[row, a:b] = mask
    z[-2, np.random.default_rng(1).random(vocab) < 0.5] = mask
    z[-2, :vocab // 2] = -np.inf                                             # both kinds of mask in a row, each with lanes of its own
    z[-2, vocab // 2:vocab - 4] = mask
    z = torch.from_numpy(z).to(t).to(gu.DEV)
    t64, _ = tokens_of(z.shape[0], vocab, 32)
    check(kind, z, t64, 5)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [40, 700, 9001, 40000])
@pytest.mark.parametrize("size", [5e6, 5.8e6, 8.4e6, 1.2e7, 1e8, 1e9, 1e10, 1e12, 1e20, 1e30, 2.2e38, 2.4e38])
def test_rows_whose_largest_is_far_from_zero(kind, vocab, size):
    """All of one value, of a few neighbouring ones, with ordinary logits below or a mask of the same size, rising and falling over every power on the way."""
    t = TYPES[kind][1]
    place = np.arange(vocab, dtype=np.float64)
    unit = size * 2.0 ** -7
    path = np.sign(place - vocab / 2) * np.minimum(2.0 ** (np.abs(place - vocab / 2) * 250 / vocab), size)
    z = np.stack([np.full(vocab, size), np.full(vocab, -size), size - unit * (place % 4), -size - unit * (place % 4), np.where(place % 3 == 0, -size, place % 5),
                  np.where(place == vocab - 3, size, -size), size - place % 7, -size - place % 7, path, path[::-1], np.where(place < 30, -size, -np.inf)])
    z = torch.from_numpy(z).to(t).to(gu.DEV).contiguous()
    t64, _ = tokens_of(z.shape[0], vocab, 33)
    check(kind, z, t64, 5)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab", [(300, 33000), (4200, 3000)])
def test_many_rows_with_a_finite_mask(kind, rows, vocab):
    """Rows of one wave with several rounds, and of the waves of a block: masks of every size in turn, in whole rounds and value by value."""
    t = TYPES[kind][1]
    z = synth.normal((rows, vocab), 34, std=3.0)
    masks = np.float64([-1e9, -1e10, -1e20, -1e30, -1e12, -np.inf])[np.arange(rows) % 6]
    place, r = np.arange(vocab), np.arange(rows)[:, None]
    z = np.where((place // 1024 + r) % 3 == 0, masks[:, None], np.where((place + r) % 7 == 0, masks[:, None], z))
    z[5::16] = masks[5::16, None]                                            # rows masked entirely
    z = torch.from_numpy(z).to(t).to(gu.DEV)
    t64, _ = tokens_of(rows, vocab, 35)
    check(kind, z, t64, 5)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [700, 9001, 40000])
def test_nan_and_infinity_beside_a_finite_mask(kind, vocab):
    dtype, t, _ = TYPES[kind]
    z = synth.normal((6, vocab), 36, std=3.0)
    z[:, 16:600] = -1e10
    z[1, 300], z[2, 300], z[3] = np.nan, np.inf, -1e20
    z[3, 5], z[4, vocab - 1] = np.nan, np.inf
    z = torch.from_numpy(z).to(t).to(gu.DEV)
    tokens = gu.dev(np.full(6, 20, np.int32))
    for top in (0, 3):
        _, (lp, ent, lse), ids, _ = run(dtype, z, tokens, vocab, top)
        for x in (lp, ent, lse):
            assert x[1:5].isnan().all() and x[[0, 5]].isfinite().all()
        if top:
            assert ids[2, 0] == 300 and ids[4, 0] == vocab - 1 and 300 not in ids[1] and 5 not in ids[3]
