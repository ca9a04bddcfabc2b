"""GPU parity of the token log probabilities (entropy, alternatives, gradient) against oracle/token_ops.py in float64.

Tolerances count roundings of u = 2^-24 (fp32).  An exponential of a distance d carries 3|d| + 4 of them (the distance, its product with log2 e, the
instruction), weighted sums of them at most 40 more in a block's order, so that log S is off by at most (40 + 4 + 3 E|d|) u, E over p, and E|d| is
at most log(vocab) + 1 for the distances from the maximum; lse adds one rounding of its own size.  bf16 stores add half a step, 2^-8."""
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
# one token to several slices, odd widths, widths at the edges of a block's registers and of a slice
SHAPES = [(1, 1), (2, 2), (3, 7), (5, 100), (2, 511), (3, 1000), (2, 2048), (2, 2049), (1, 4097), (2, 8192), (2, 8193), (1, 16391), (3, 50021), (1, 131072),
          (300, 33)]


def tol(vocab):
    return (48 + 4 * (np.log(vocab) + 2)) * U


def f64(t):
    return t.double().cpu().numpy()


def logits_of(rows, vocab, seed, dtype, pad=0, offset=0, masked=0.0, std=3.0):
    whole = torch.full((rows * (vocab + pad) + offset,), float("nan"), dtype=dtype, device=gu.DEV)
    view = whole[offset:].view(rows, vocab + pad)[:, :vocab]
    z = synth.normal((rows, vocab), seed, std=std)
    if masked:
        z[np.random.default_rng(seed).random((rows, vocab)) < masked] = -np.inf
    view.copy_(torch.from_numpy(z))
    return view, view.double().cpu().numpy()


def tokens_of(rows, vocab, seed):
    t = np.random.default_rng(seed).integers(0, vocab, rows)
    if rows > 2:
        t[1], t[2] = -1, vocab                      # two kinds of positions that do not count
    return t, gu.dev(t.astype(np.int32))


def run(dtype, z, tokens, vocab, top=0):
    rows = z.shape[0]
    d = lc.TokenDesc(rows, vocab, ld=z.stride(0) if rows > 1 else 0, dtype=dtype, top=top)
    out = [gu.guarded((rows,), torch.float32) for _ in range(3)]
    ids = gu.guarded((rows, top), torch.float32) if top else None
    lps = gu.guarded((rows, top), torch.float32) if top else None
    lc.token_logprob_fwd(d, z, tokens, out[0][0], out[1][0], out[2][0], ids[0] if top else None, lps[0] if top else None,
                         gu.workspace(lc.token_logprob_workspace_bytes(d)))
    torch.cuda.synchronize()
    for _, check in out + ([ids, lps] if top else []):
        check()
    return d, [o for o, _ in out], ids[0].view(torch.int32).cpu().numpy() if top else None, f64(lps[0]) if top else None


def close(got, want, bound):
    fine = np.isfinite(want)
    return np.array_equal(got[~fine], want[~fine]) and np.all(np.abs(got[fine] - want[fine]) <= np.broadcast_to(bound, want.shape)[fine])


def check_forward(vocab, got, want, top):
    (lp, ent, lse), ids, lps = [f64(x) for x in got[1]], got[2], got[3]
    wlp, went, wlse, wids, wlps = want
    e = tol(vocab)
    assert close(lp, wlp, e + 3 * U * np.abs(wlp))
    assert close(lse, wlse, e + U * np.abs(wlse))
    assert close(ent, went, 2 * e + 4 * U * went + e * went)
    if top:
        assert np.array_equal(ids, wids)
        assert close(lps, wlps, e + 3 * U * np.abs(wlps))


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab", SHAPES)
@pytest.mark.parametrize("top", [0, 1, 5, 32])
@pytest.mark.parametrize("pad,offset,masked", [(0, 0, 0.0), (5, 1, 0.4)])
def test_forward(kind, rows, vocab, top, pad, offset, masked):
    dtype, t, _ = TYPES[kind]
    z, z64 = logits_of(rows, vocab, 1, t, pad, offset, masked)
    t64, tokens = tokens_of(rows, vocab, 2)
    got = run(dtype, z, tokens, vocab, top)
    check_forward(vocab, got, ops.token_logprob(z64, t64, top), top)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [40, 700, 5000, 30000])
@pytest.mark.parametrize("case", ["equal", "falling", "rising", "two_values", "one_lane", "all_masked", "one_left", "lowest", "large"])
def test_alternatives_of_unusual_rows(kind, vocab, case):
    """Equal values (more than there is room for), orders that put the largest into one lane or slice, masks that leave nothing or one, the
    type's lowest value in place of a mask, logits far from zero."""
    dtype, t, _ = TYPES[kind]
    rows, top = 2, 20
    place = np.arange(vocab, dtype=np.float64)
    z = {"equal": np.full(vocab, 1.5), "falling": -place / 64, "rising": place / 64, "two_values": np.where(place % 3 == 1, 2.0, -1.0),
         "one_lane": np.where(place % 2048 < 8, 5 + place / 4096, -place / 4096), "all_masked": np.full(vocab, -np.inf),
         "one_left": np.where(place == vocab - 2, -7.0, -np.inf), "lowest": np.where(place % 5 == 0, place / 512, float(torch.finfo(t).min)),
         "large": 3e4 + place % 17}[case]
    z = torch.from_numpy(np.stack([z, z[::-1]])).to(t).to(gu.DEV).contiguous()
    t64, tokens = np.array([0, vocab - 1]), gu.dev(np.array([0, vocab - 1], np.int32))
    got = run(dtype, z, tokens, vocab, top)
    check_forward(vocab, got, ops.token_logprob(f64(z), t64, top), top)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [50, 20000])
def test_nan_and_infinity_stay_in_their_rows(kind, vocab):
    dtype, t, _ = TYPES[kind]
    z, _ = logits_of(4, vocab, 3, t)
    z[1, vocab // 2] = float("nan")
    z[2, 3] = float("inf")
    tokens = gu.dev(np.array([1, 2, 4, 5], np.int32))
    d, (lp, ent, lse), ids, lps = run(dtype, z, tokens, vocab, 3)
    for x in (lp, ent, lse):
        assert x[[1, 2]].isnan().all() and x[[0, 3]].isfinite().all()
    assert ids[2, 0] == 3 and vocab // 2 not in ids[1] and np.isnan(lps[[1, 2]]).all() and np.isfinite(lps[[0, 3]]).all()
    dz, one = torch.empty_like(z), torch.ones(4, device=gu.DEV)
    lc.token_logprob_bwd(d, z, tokens, lse, ent, one, one, dz)
    torch.cuda.synchronize()
    assert dz[[1, 2]].isnan().all() and dz[[0, 3]].isfinite().all()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab", SHAPES)
@pytest.mark.parametrize("parts", ["both", "logprob", "entropy"])
def test_backward(kind, rows, vocab, parts):
    dtype, t, half = TYPES[kind]
    pad = vocab % 4
    z, z64 = logits_of(rows, vocab, 4, t, pad, pad, 0.2 if vocab > 50 else 0.0)
    t64, tokens = tokens_of(rows, vocab, 5)
    d, (lp, ent, lse), _, _ = run(dtype, z, tokens, vocab)
    a64, b64 = np.float32([0.5 + i % 3 for i in range(rows)]), np.float32([-0.25 * (1 + i % 2) for i in range(rows)])
    a64, b64 = (a64 if parts != "entropy" else 0 * a64), (b64 if parts != "logprob" else 0 * b64)
    whole, check = gu.guarded((rows, vocab + 3), t, offset=2 * pad * (2 if kind == "f32" else 1))
    before = whole.clone()
    lc.token_logprob_bwd(d, z, tokens, lse, ent if parts != "logprob" else None, gu.dev(a64) if parts != "entropy" else None,
                         gu.dev(b64) if parts != "logprob" else None, whole, dlogits_ld=vocab + 3)
    torch.cuda.synchronize()
    check()
    dz = f64(whole[:, :vocab])
    assert whole[:, vocab:].isnan().all() and before.isnan().all()           # the pad is not written
    want = ops.token_logprob_bwd(z64, t64, a64.astype(np.float64), b64.astype(np.float64))
    _, e64, l64, _, _ = ops.token_logprob(z64, t64)
    d64 = np.where(np.isfinite(z64), np.abs(z64 - l64[:, None]), 0.0)
    p = np.where(np.isfinite(z64), np.exp(-d64), 0.0)
    size = p * (np.abs(a64)[:, None] + np.abs(b64)[:, None] * (d64 + e64[:, None]))
    # p by the rounding of lse, of the distance and of the exponential; the entropy's and the token's own term besides
    bound = size * (tol(vocab) + U * (np.abs(l64)[:, None] + 3 * d64 + 8)) + p * np.abs(b64)[:, None] * (2 * tol(vocab) + 5 * U * e64[:, None]
            + tol(vocab) * e64[:, None] + U * np.abs(l64)[:, None]) + U * np.abs(a64)[:, None]
    assert np.all(np.abs(dz - want) <= half * (1 + half) * np.abs(want) + (1 + half) * bound)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [7, 700, 9001])
def test_rows_far_from_zero_and_rows_of_the_lowest_value(kind, vocab):
    """Where products with log2 e overflow (the type's lowest and highest value) and where lse as stored says little (|lse| of 3e4 to 3e38): log p stays
    what the differences of the logits give.  On such rows p is exp(d - log S) with d exact or rounded once, so that the gradient is within tol + 4|d| u of it,
    and half a unit of lse's own size where it is formed from lse: 2^-24 * 256 in fp32, 2^-24 * 16384 in bf16."""
    dtype, t, half = TYPES[kind]
    low, high = float(torch.finfo(t).min), float(torch.finfo(t).max)
    place = np.arange(vocab, dtype=np.float64)
    z = np.stack([np.full(vocab, low), np.where(place % 3 == 0, low, place % 5), np.where(place == 2, high, low), -3e4 - place % 7, 250.0 + place % 4, 7e3 + place % 4,
                  np.where(place < 3, -np.inf, low)])
    z = torch.from_numpy(z).to(t).to(gu.DEV)
    rows = z.shape[0]
    t64 = np.array([vocab // 2] * rows)
    tokens = gu.dev(t64.astype(np.int32))
    d, (lp, ent, lse), ids, lps = run(dtype, z, tokens, vocab, 3)
    in_range = lambda a: np.where(np.abs(a) > np.finfo(np.float32).max, np.copysign(np.inf, a), a)      # (the highest above the lowest: beyond fp32)
    check_forward(vocab, (d, (lp, ent, lse), ids, lps), [in_range(a) for a in ops.token_logprob(f64(z), t64, 3)], 3)
    d, (lp2, ent2, lse2), _, _ = run(dtype, z, tokens, vocab)
    check_forward(vocab, (d, (lp2, ent2, lse2), None, None), [in_range(a) for a in ops.token_logprob(f64(z), t64, 0)], 0)
    dz, one = torch.empty_like(z), torch.ones(rows, device=gu.DEV)
    lc.token_logprob_bwd(d, z, tokens, lse, ent, one, 0.5 * one, dz)
    torch.cuda.synchronize()
    w64, e64, _, _, _ = ops.token_logprob(f64(z), t64)
    m = np.max(f64(z), axis=1, keepdims=True)
    logp = (f64(z) - m) - np.log(np.sum(np.exp(f64(z) - m), axis=1, keepdims=True))
    p, fine = np.exp(logp), np.where(np.exp(logp) > 0, logp, 0.0)
    want = (place == vocab // 2) - p - 0.5 * p * (fine + e64[:, None])
    rel = tol(vocab) * (2 + e64[:, None]) + U * (4 * np.abs(fine) + (16384 if kind == "bf16" else 256))
    bound = p * (1.5 + np.abs(fine) + e64[:, None]) * rel + 2 * U
    assert np.all(np.abs(f64(dz) - want) <= half * (1 + half) * np.abs(want) + (1 + half) * bound)


def test_the_gradient_against_differences():
    """Central differences of the float64 sum over the kernel's own forward outputs, fp32: a step of 2^-6 keeps its rounding under 1e-3."""
    z = synth.normal((2, 50), 6)
    tokens, a, b = gu.dev(np.array([7, 49], np.int32)), np.float32([1.0, -0.5]), np.float32([0.5, 2.0])
    forward = lambda y: sum(float(np.dot(f64(o), c)) for o, c in zip(run(lc.LC_F32, gu.dev(y), tokens, 50)[1][:2], (a, b)))
    d, (lp, ent, lse), _, _ = run(lc.LC_F32, gu.dev(z), tokens, 50)
    dz = torch.empty((2, 50), device=gu.DEV)
    lc.token_logprob_bwd(d, gu.dev(z), tokens, lse, ent, gu.dev(a), gu.dev(b), dz)
    got = f64(dz)
    for i, j in [(0, 7), (0, 0), (1, 49), (1, 20)]:
        up, down = z.copy(), z.copy()
        up[i, j] += np.float32(2.0 ** -6)
        down[i, j] -= np.float32(2.0 ** -6)
        numeric = (forward(up) - forward(down)) / float(up[i, j].astype(np.float64) - down[i, j].astype(np.float64))
        assert abs(numeric - got[i, j]) < 1e-3


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_gradient_in_the_logits_own_buffer_on_another_stream(kind):
    dtype, t, _ = TYPES[kind]
    rows, vocab = 40, 1001
    z, _ = logits_of(rows, vocab, 7, t)
    _, tokens = tokens_of(rows, vocab, 8)
    d, (lp, ent, lse), _, _ = run(dtype, z, tokens, vocab)
    one, dz, side = torch.ones(rows, device=gu.DEV), torch.empty_like(z), torch.cuda.Stream()
    lc.token_logprob_bwd(d, z, tokens, lse, ent, one, one, dz)
    torch.cuda.synchronize()
    lc.token_logprob_bwd(d, z, tokens, lse, ent, one, one, z, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(z, dz)


def test_many_rows_of_one_element_and_bit_identical_reruns():
    z, _ = logits_of(3000, 9000, 9, torch.bfloat16)
    _, tokens = tokens_of(3000, 9000, 10)
    first, again = run(lc.LC_BF16, z, tokens, 9000, 8), run(lc.LC_BF16, z, tokens, 9000, 8)
    assert all(torch.equal(x, y) for x, y in zip(first[1], again[1])) and np.array_equal(first[2], again[2]) and np.array_equal(first[3], again[3])


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [700, 9001, 60000])
def test_gradient_of_rows_far_from_zero_in_the_logits_own_buffer(kind, vocab):
    """Rows whose sums the gradient makes again (see the lowest value and |lse| above): no part of them may be written before they are read."""
    dtype, t, _ = TYPES[kind]
    rows = 24
    place = np.arange(vocab, dtype=np.float64)
    z = np.stack([3e4 * (1 + r) + (place * (r + 3)) % 11 if r % 3 else np.where(place % 7 == r % 7, float(torch.finfo(t).max), float(torch.finfo(t).min)) for r in range(rows)])
    z = torch.from_numpy(z).to(t).to(gu.DEV)
    _, tokens = tokens_of(rows, vocab, 11)
    d, (lp, ent, lse), _, _ = run(dtype, z, tokens, vocab)
    one, dz = torch.ones(rows, device=gu.DEV), torch.empty_like(z)
    lc.token_logprob_bwd(d, z, tokens, lse, ent, one, one, dz)
    lc.token_logprob_bwd(d, z, tokens, lse, ent, one, one, z)
    torch.cuda.synchronize()
    assert torch.equal(z, dz)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab", [(70, 34001), (130, 66005), (270, 9001), (300, 33000), (1100, 16003), (4200, 1500), (2, 270001)])
@pytest.mark.parametrize("top", [0, 5])
def test_forward_with_rows_divided_in_every_way(kind, rows, vocab, top):
    """Rows by one wave, by two to sixteen of a block, and by blocks of one; one round a wave and several; by a third of the rows with masked logits."""
    dtype, t, _ = TYPES[kind]
    z, _ = logits_of(rows, vocab, 12, t, pad=vocab % 8)
    z[::3, vocab // 7: vocab // 2] = -float("inf")
    z64 = f64(z)
    t64, tokens = tokens_of(rows, vocab, 13)
    d, got, ids, lps = run(dtype, z, tokens, vocab, top)
    check_forward(vocab, (d, got, ids, lps), ops.token_logprob(z64, t64, top), top)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("top", [0, 3])
def test_more_rows_than_a_grid_takes_at_once(kind, top):
    rows, vocab = 70001, 17
    dtype, t, half = TYPES[kind]
    z, z64 = logits_of(rows, vocab, 14, t, masked=0.2)
    t64, tokens = tokens_of(rows, vocab, 15)
    d, (lp, ent, lse), ids, lps = run(dtype, z, tokens, vocab, top)
    want = ops.token_logprob(z64, t64, top)
    check_forward(vocab, (d, (lp, ent, lse), ids, lps), want, top)
    one, dz = torch.ones(rows, device=gu.DEV), torch.empty_like(z)
    lc.token_logprob_bwd(d, z, tokens, lse, None, one, None, dz)
    torch.cuda.synchronize()
    exact = ops.token_logprob_bwd(z64, t64, np.ones(rows), np.zeros(rows))
    assert np.all(np.abs(f64(dz) - exact) <= half * (1 + half) * np.abs(exact) + (1 + half) * (tol(vocab) + 16 * U))


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [40000, 70000, 140000, 300000])
@pytest.mark.parametrize("top", [20, 32])
@pytest.mark.parametrize("case", ["equal", "two_values", "falling", "rising", "few_steps", "one_block"])
def test_alternatives_joined_from_many_lists(kind, vocab, top, case):
    """Rows in 40 to 293 blocks whose lists together hold more equal or near-equal keys than there is room for at once (256), one list a lane and several."""
    dtype, t, _ = TYPES[kind]
    place = np.arange(vocab, dtype=np.float64)
    z = {"equal": np.full(vocab, 1.5), "two_values": np.where(place % 3 == 1, 2.0, -1.0), "falling": -np.floor(place / 64) / 64, "rising": np.floor(place / 64) / 64,
         "few_steps": np.floor(place / vocab * 7), "one_block": np.where(place // 1024 == 2, 2.0, 1.0)}[case]
    z = torch.from_numpy(np.stack([z, z[::-1]])).to(t).to(gu.DEV).contiguous()
    t64 = np.array([0, vocab - 1])
    got = run(dtype, z, gu.dev(t64.astype(np.int32)), vocab, top)
    check_forward(vocab, got, ops.token_logprob(f64(z), t64, top), top)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab", [(64, 40000), (64, 50021), (96, 98304), (16, 33000)])
@pytest.mark.parametrize("top", [17, 20, 32])
def test_alternatives_joined_from_few_more_lists_than_places(kind, rows, vocab, top):
    """20 to 33 lists: nearly as many as places, where a bound that every list has to reach would be the least of all; a third of the rows with one list's worth of logits, so that most
    lists hold less than they answer for."""
    dtype, t, _ = TYPES[kind]
    z, _ = logits_of(rows, vocab, 16, t, masked=0.1)
    z[::3] = torch.where(torch.arange(vocab, device=gu.DEV) % 2003 < 2, z[::3], torch.tensor(-float("inf"), dtype=t, device=gu.DEV))
    z[1::6, 5000:9000] = 2.5
    t64, tokens = tokens_of(rows, vocab, 17)
    check_forward(vocab, run(dtype, z, tokens, vocab, top), ops.token_logprob(f64(z), t64, top), top)
