"""The token model's output side as one path (paper_1709_05011_amd/token_head_step.py) against the float64 definitions chained with numpy products, its
training, and its capture in a HIP graph."""
import numpy as np
import pytest
import torch

from oracle import token_ops as ops
from paper_1709_05011_amd import larsconv as lc
from paper_1709_05011_amd import synth
from paper_1709_05011_amd.token_head_step import TokenHeadStep

import gpu_util as gu

pytestmark = pytest.mark.gpu
# relative to the largest value of each tensor: fp32 products over 64 to 96 columns and 300 tokens stay under 1e-4 of it (the parity bound of the
# convolutions); bf16 rounds y, the logits, their gradient and dy once each (2^-8 of the value, |logits| about 8 and weights of order 1 behind them): 5 %
TOL = {"f32": 1e-4, "bf16": 0.05}
f64 = lambda t: t.double().cpu().numpy()


def setup(kind, rows, width, vocab, **kw):
    t = torch.bfloat16 if kind == "bf16" else torch.float32
    head = TokenHeadStep(width, vocab, lc.LC_BF16 if kind == "bf16" else lc.LC_F32, **kw)
    head.load(gu.dev(synth.normal((vocab, width), 1, std=2.0 / np.sqrt(width))), gu.dev(1 + synth.normal((width,), 2, std=0.2)))
    x, r = (gu.dev(synth.normal((rows, width), s)).to(t) for s in (3, 4))
    tokens = np.random.default_rng(5).integers(0, vocab, rows)
    tokens[0] = -1
    return head, x, r, tokens, gu.dev(tokens.astype(np.int32))


def chain(head, x, r, tokens, a, b, kind):
    """The same in float64 from the values the device holds."""
    store = (lambda v: ops.bf16(v.astype(np.float32))) if kind == "bf16" else (lambda v: v)
    w, gamma = f64(head.params["w"] if head.w_lowp is None else head.w_lowp)[:head.vocab], f64(head.params["gamma"])
    h, rstd, y = ops.rmsnorm(f64(x), f64(r), gamma, 1e-5, store)
    z = y @ w.T
    lp, ent, _, ids, top = ops.token_logprob(z, tokens, 5)
    dz = ops.token_logprob_bwd(z, tokens, a, b)
    dx, dgamma = ops.rmsnorm_bwd(h, rstd, gamma, dz @ w)
    return lp, ent, ids, top, dx, dz.T @ y, dgamma


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rows,width,vocab", [(1, 64, 40), (7, 96, 1003), (300, 64, 517)])
def test_score_and_step(kind, rows, width, vocab):
    head, x, r, tokens, dev_tokens = setup(kind, rows, width, vocab)
    a, b = np.full(rows, -1.0 / rows), np.full(rows, -0.05 / rows)
    lp, ent, ids, top, dx, dw, dgamma = chain(head, x, r, tokens, a, b, kind)
    near = lambda got, want: float(np.max(np.abs(f64(got) - want))) <= TOL[kind] * max(1e-12, float(np.max(np.abs(want))))
    got = head.score(x, r, dev_tokens, top=5)
    torch.cuda.synchronize()
    assert near(got[0], lp) and near(got[1], ent) and near(got[3], top)
    before = {k: p.clone() for k, p in head.params.items()}
    got = head.step(x, r, dev_tokens, gu.dev(np.float32(a)), gu.dev(np.float32(b)))
    torch.cuda.synchronize()
    assert near(got[0], lp) and near(got[1], ent) and near(got[2], dx)
    assert near(head.grads["w"][:vocab], dw) and near(head.grads["gamma"], dgamma) and not head.grads["w"][vocab:].any()
    for k, decay in (("w", 0.1), ("gamma", 0.0)):             # the update by the gradients the device made
        g = f64(head.grads[k])
        want, _, _ = ops.adamw(f64(before[k]), g, 0 * g, 0 * g, 1e-3, 0.9, 0.95, 1e-8, decay, 1)
        assert np.max(np.abs(f64(head.params[k]) - want)) < 1e-5 * 1e-3 + 2.0 ** -22 * np.max(np.abs(want))
    if head.w_lowp is not None:
        assert torch.equal(head.w_lowp, head.params["w"].bfloat16())


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("states_in_8_bits", [False, True])
def test_training_learns_the_tokens(kind, states_in_8_bits):
    """64 tokens of their own hidden states: forty steps bring the mean log probability from under -4 to over -1, with states of either width."""
    rows = 64
    head, x, r, tokens, dev_tokens = setup(kind, rows, 128, 200, states_in_8_bits=states_in_8_bits, lr=0.02)
    a = torch.full((rows,), -1.0 / rows, device=gu.DEV)
    first = f64(head.score(x, r, dev_tokens)[0])[1:].mean()
    for _ in range(40):
        head.step(x, r, dev_tokens, a)
    last = f64(head.score(x, r, dev_tokens)[0])[1:].mean()
    assert first < -4 and last > -1, (first, last)


def test_packed():
    head, x, r, _, _ = setup("bf16", 9, 200, 40)
    total, codes, scales = head.packed(x, r)
    torch.cuda.synchronize()
    h, _, y = ops.rmsnorm(f64(x), f64(r), f64(head.params["gamma"]), 1e-5, lambda v: ops.bf16(v.astype(np.float32)))
    assert np.array_equal(f64(total), h) and scales.shape == (9, 2)
    back = codes.float().double().cpu().numpy() * np.repeat(f64(scales), 128, axis=1)[:, :200]
    assert np.max(np.abs(back - y)) < 2.0 ** -4 * 1.001 * np.max(np.abs(y))


@pytest.mark.parametrize("states_in_8_bits", [False, True])
def test_the_step_in_a_graph(states_in_8_bits):
    """Captured once and replayed with eager work between: every replay from the same start gives the eager step's bits."""
    rows = 50
    head, x, r, tokens, dev_tokens = setup("bf16", rows, 128, 9000, states_in_8_bits=states_in_8_bits)
    a, b = torch.full((rows,), -1.0 / rows, device=gu.DEV), torch.full((rows,), -0.01 / rows, device=gu.DEV)
    state = [*head.params.values(), *head.m, *head.v, head.w_lowp] + ([*head.m_scale, *head.v_scale] if states_in_8_bits else [])
    start = [t.clone() for t in state]

    def restore():
        for t, s in zip(state, start):
            t.copy_(s)
        head.steps = 0

    def results():
        torch.cuda.synchronize()
        return [t.clone() for t in (*state, *out, *head.grads.values())]

    out = head.step(x, r, dev_tokens, a, b)
    want = results()
    side = torch.cuda.Stream()
    restore()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        head.step(x, r, dev_tokens, a, b)
    for _ in range(3):
        restore()
        junk = [torch.randn(1000, 1000, device=gu.DEV) @ torch.randn(1000, 1000, device=gu.DEV) for _ in range(3)]
        for t in (*out, *head.grads.values()):
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        assert all(torch.equal(g, w) for g, w in zip(results(), want))
        del junk


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_ragged_calls_in_shared_room(kind):
    """Calls of many sizes, rising and falling, with steps between: each gives the bits that an object of its own gives."""
    rows, width, vocab = 40, 64, 1003
    head, x, r, _, tokens = setup(kind, rows, width, vocab, lr=0.0)
    alone = lambda: setup(kind, rows, width, vocab, lr=0.0)[0]
    a = torch.full((rows,), -1.0 / rows, device=gu.DEV)
    for n, top in [(3, 0), (17, 5), (1, 5), (40, 0), (2, 20), (39, 0), (5, 1), (6, 1), (7, 1), (8, 1), (9, 1), (3, 0), (40, 3)]:
        got = [None if t is None else t.clone() for t in head.score(x[:n], r[:n], tokens[:n], top=top)]
        want = alone().score(x[:n], r[:n], tokens[:n], top=top)
        assert all(p is q or torch.equal(p, q) for p, q in zip(got, want)), (n, top)
        other = alone()
        got = [t.clone() for t in head.step(x[:n], r[:n], tokens[:n], a[:n])] + [g.clone() for g in head.grads.values()]
        want = list(other.step(x[:n], r[:n], tokens[:n], a[:n])) + list(other.grads.values())
        assert all(torch.equal(p, q) for p, q in zip(got, want)), n


@pytest.mark.parametrize("warm", [True, False])
def test_a_graph_keeps_what_it_works_in(warm):
    """A step recorded with or without an eager call of its size before; later calls of other sizes, the larger ones in a new room, take nothing from it."""
    rows, width, vocab = 16, 64, 1003
    head, x, r, _, tokens = setup("bf16", 50, width, vocab, lr=0.0)
    a = torch.full((50,), -1.0 / rows, device=gu.DEV)
    call = lambda n: head.step(x[:n], r[:n], tokens[:n], a[:n])
    want = [t.clone() for t in call(rows)] + [g.clone() for g in head.grads.values()]
    if not warm:
        head, _, _, _, _ = setup("bf16", 50, width, vocab, lr=0.0)
        torch.cuda.synchronize()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        out = call(rows)
        again = call(rows)
    assert all(p is q for p, q in zip(out, again))
    for n in (50, 1, 3, 7, 20, 50, 9, 11, 13, 21, 2, 16):
        call(n)
        head.score(x[:n], r[:n], tokens[:n], top=3)
        junk = [torch.full((k,), float("nan"), device=gu.DEV) for k in (1 << 14, 1 << 16, 1 << 18, 1 << 20)]      # what an eager call freed is written by others
        for t in (*out, *head.grads.values()):
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip([*out, *head.grads.values()], want)), n
        del junk


def test_calls_on_streams_in_turn():
    """A step behind long work on one stream, a score and a step on two others, with nothing between them: each sees what the one before it has left."""
    rows, width, vocab = 30, 64, 1003
    a = torch.full((rows,), -1.0 / rows, device=gu.DEV)

    def run(streams, busy):
        head, x, r, _, tokens = setup("bf16", rows, width, vocab, lr=0.01)
        out = []
        torch.cuda.synchronize()
        for i, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                for _ in range(busy):
                    torch.mm(big, big)
                if i % 2:
                    out += [t.clone() for t in head.score(x[:rows - i], r[:rows - i], tokens[:rows - i], top=i)]
                else:
                    out += [t.clone() for t in head.step(x, r, tokens, a)]
            busy = max(busy - 10, 0)
        torch.cuda.synchronize()
        return out + [p.clone() for p in head.params.values()]

    big = torch.randn(4096, 4096, device=gu.DEV)
    side = [torch.cuda.Stream() for _ in range(2)]
    want = run([torch.cuda.current_stream()] * 9, 0)
    got = run([side[0], torch.cuda.current_stream(), side[1], side[0], torch.cuda.current_stream(), side[1], side[1], side[0], torch.cuda.current_stream()], 30)
    assert all(torch.equal(p, q) for p, q in zip(got, want))


@pytest.mark.parametrize("states_in_8_bits", [False, True])
def test_a_step_over_no_rows(states_in_8_bits):
    """Gradients are zero: the classifier decays, the norm's scale stays, and a step over rows after it is the second step."""
    head, x, r, _, tokens = setup("bf16", 20, 64, 40, states_in_8_bits=states_in_8_bits, lr=0.25)
    a = torch.full((20,), -0.05, device=gu.DEV)
    before = {k: p.clone() for k, p in head.params.items()}
    lp, ent, dx = head.step(x[:0], r[:0], tokens[:0], a[:0])
    torch.cuda.synchronize()
    assert lp.shape == ent.shape == (0,) and dx.shape == (0, 64) and head.steps == 1
    assert torch.equal(head.params["gamma"], before["gamma"]) and not any(g.any() for g in head.grads.values())
    want = before["w"].double() * (1 - float(np.float32(0.25 * 0.1)))
    assert bool(((head.params["w"].double() - want).abs() <= 2.0 ** -24 * want.abs()).all()) and torch.equal(head.w_lowp, head.params["w"].bfloat16())
    head.step(x, r, tokens, a)
    torch.cuda.synchronize()
    assert head.steps == 2 and all(p.isfinite().all() for p in head.params.values()) and head.grads["w"].any()
