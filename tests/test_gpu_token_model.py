"""A whole step of a token model (paper_1709_05011_amd/token_model_step.py): its log probabilities and gradients against the same model in float64, its updates against the oracle's by
the gradients that it made, and its capture in a HIP graph."""
import numpy as np
import pytest
import torch

from oracle import token_model_ops as ops
from oracle import token_ops
from paper_1709_05011_amd import larsconv as lc
from paper_1709_05011_amd import synth
from paper_1709_05011_amd.token_model_step import TokenModelStep

import gpu_util as gu

pytestmark = pytest.mark.gpu
# relative to the largest value of each tensor: fp32 products over 48 to 96 columns and 300 tokens stay under 1e-4 of it (the parity bound of the convolutions).  bf16: each of a block's
# four stores and of the four around them is off by 2^-9 of a value in the mean square, forward and backward: 2 * 12 stores of two blocks, which add up as roots, and at worst all of one sign 24 * 2^-9
TOL = {"f32": 1e-4, "bf16": 0.05}
f64 = lambda t: t.double().cpu().numpy()


def setup(kind, rows, width, vocab, blocks, **kw):
    model = TokenModelStep(width, vocab, blocks, lc.LC_BF16 if kind == "bf16" else lc.LC_F32, **kw)
    params = {"table": synth.normal((vocab, width), 1, std=1.0 / np.sqrt(width))}
    for l in range(blocks):
        params |= {f"gamma{l}": 1 + synth.normal((width,), 10 * l + 2, std=0.2), f"beta{l}": synth.normal((width,), 10 * l + 3, std=0.2),
                   f"w{l}": synth.normal((width, width), 10 * l + 4, std=1.0 / np.sqrt(width))}
    model.load({k: gu.dev(v) for k, v in params.items()}, gu.dev(synth.normal((vocab, width), 5, std=2.0 / np.sqrt(width))), gu.dev(1 + synth.normal((width,), 6, std=0.2)))
    rng = np.random.default_rng(7)
    tokens, targets = rng.integers(0, vocab, rows).astype(np.int32), rng.integers(0, vocab, rows).astype(np.int32)
    tokens[rows // 2], targets[0] = -1, -1
    return model, tokens, targets


def in_64_bits(model, tokens, targets, a):
    """(log probabilities, gradients by name, the head's) of the values that the device computes with, by torch's float64 on the CPU."""
    leaf = lambda t: t.double().cpu().requires_grad_()
    p = {k: leaf(model.lowp.get(k, v)) for k, v in model.params.items()}
    head = {"w": leaf((model.head.params["w"] if model.head.w_lowp is None else model.head.w_lowp)[:model.vocab]), "gamma": leaf(model.head.params["gamma"])}
    t, goal = torch.from_numpy(tokens).long(), torch.from_numpy(targets).long()
    stream = torch.where((t >= 0)[:, None], model.scale * p["table"][t.clamp(min=0)], 0.0)
    for l in range(model.blocks):
        mean = stream.mean(1, keepdim=True)
        n = (stream - mean) / torch.sqrt(((stream - mean) ** 2).mean(1, keepdim=True) + model.eps)
        stream = stream + (n * p[f"gamma{l}"] + p[f"beta{l}"]) @ p[f"w{l}"].T
    y = stream / torch.sqrt((stream ** 2).mean(1, keepdim=True) + model.eps) * head["gamma"]
    logp = torch.log_softmax(y @ head["w"].T, 1)
    logprob = torch.where(goal >= 0, logp.gather(1, goal.clamp(min=0)[:, None])[:, 0], 0.0)
    (logprob * torch.from_numpy(a)).sum().backward()
    return logprob.detach().numpy(), {k: v.grad.numpy() for k, v in p.items()}, {k: v.grad.numpy() for k, v in head.items()}


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rows,width,vocab,blocks", [(1, 64, 40, 1), (7, 96, 1003, 2), (300, 48, 517, 2), (5000, 64, 100, 1), (33, 64, 70, 0)])
def test_a_step(kind, rows, width, vocab, blocks):
    model, tokens, targets = setup(kind, rows, width, vocab, blocks)
    a = np.full(rows, -1.0 / rows)
    logprob, grads, head_grads = in_64_bits(model, tokens, targets, a)
    near = lambda got, want: float(np.max(np.abs(f64(got) - want))) <= TOL[kind] * max(1e-12, float(np.max(np.abs(want))))
    dev_tokens, dev_targets = gu.dev(tokens), gu.dev(targets)
    assert near(model.score(dev_tokens, dev_targets, top=3)[0], logprob)
    before = {k: f64(p) for k, p in model.params.items()}
    got = model.step(dev_tokens, dev_targets, gu.dev(np.float32(a)))
    torch.cuda.synchronize()
    assert near(got[0], logprob)
    for k in grads:
        assert near(model.grads[k], grads[k]), k
    assert near(model.head.grads["w"][:vocab], head_grads["w"]) and near(model.head.grads["gamma"], head_grads["gamma"])
    for k in model.params:                                    # the updates by the gradients the device made
        g, now = f64(model.grads[k]), f64(model.params[k])
        if k.startswith("w"):
            want, _ = ops.muon(before[k], g, 0 * g, 0.02, 0.95, 0.1)
            assert np.sqrt(np.sum((now - want) ** 2)) <= 1e-4 * 0.02 * np.sqrt(width) + 2.0 ** -22 * np.sqrt(np.sum(want ** 2)), k
        else:
            want, _, _ = token_ops.adamw(before[k], g, 0 * g, 0 * g, 1e-3, 0.9, 0.95, 1e-8, 0.1 if k == "table" else 0.0, 1)
            assert np.max(np.abs(now - want)) < 1e-5 * 1e-3 + 2.0 ** -22 * np.max(np.abs(want)), k
    for k, c in model.lowp.items():
        assert torch.equal(c, model.params[k].bfloat16()), k


def test_no_rows():
    model, _, _ = setup("f32", 3, 32, 20, 2)
    none, empty = torch.empty(0, dtype=torch.int32, device=gu.DEV), torch.empty(0, device=gu.DEV)
    assert model.score(none, none)[0].shape == (0,)
    before = {k: p.clone() for k, p in model.params.items()}
    model.step(none, none, empty)
    torch.cuda.synchronize()
    assert all(not g.any() for g in model.grads.values())
    decay = {"t": 1 - 1e-3 * 0.1, "w": 1 - 0.02 * 0.1, "g": 1.0, "b": 1.0}
    for k, p in model.params.items():
        assert np.max(np.abs(f64(p) - decay[k[0]] * f64(before[k]))) <= 2.0 ** -22 * max(1e-30, float(before[k].abs().max())), k


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_the_step_in_a_graph_and_on_another_stream(kind):
    """Captured once and replayed with eager work between: every replay from the same start gives the eager step's bits; so does an eager step on another stream."""
    rows = 50
    model, tokens, targets = setup(kind, rows, 128, 900, 3)
    tokens, targets, a = gu.dev(tokens), gu.dev(targets), torch.full((rows,), -1.0 / rows, device=gu.DEV)
    state = [*model.params.values(), *model.m.values(), *model.v.values(), *model.lowp.values(), *model.head.params.values(), *model.head.m, *model.head.v]
    state += [model.head.w_lowp] if model.head.w_lowp is not None else []
    start = [t.clone() for t in state]

    def restore():
        for t, s in zip(state, start):
            t.copy_(s)
        model.steps = model.head.steps = 0

    def results(out):
        torch.cuda.synchronize()
        return [t.clone() for t in (*state, *out, *model.grads.values(), *model.head.grads.values())]

    want = results(model.step(tokens, targets, a))
    side = torch.cuda.Stream()
    restore()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out = model.step(tokens, targets, a)
    assert all(torch.equal(x, y) for x, y in zip(results(out), want))
    restore()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = model.step(tokens, targets, a)
    for _ in range(3):
        restore()
        junk = [torch.randn(1000, 1000, device=gu.DEV) @ torch.randn(1000, 1000, device=gu.DEV) for _ in range(3)]
        for g in model.grads.values():
            g.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        assert all(torch.equal(x, y) for x, y in zip(results(out), want))
        del junk
        restore()
        model.step(tokens, targets, a)
    restore()
