"""The output side of a token model refuses tensors that the entry points' pointers would misread, before any launch (no GPU needed)."""
import pytest
import torch

from paper_1709_05011_amd import larsconv as lc
from paper_1709_05011_amd.token_head_step import TokenHeadStep

ROWS, WIDTH = 4, 16


@pytest.mark.parametrize("bad", ["strided", "width", "type", "rows", "tokens64", "dlogprob_rows", "dentropy_type", "dtotal_strided"])
def test_refusals(bad):
    head = TokenHeadStep(WIDTH, 40, lc.LC_F32, device="cpu")
    x, wide = torch.zeros(ROWS, WIDTH), torch.zeros(ROWS, 2 * WIDTH)
    a = dict(x=x, residual=x, tokens=torch.zeros(ROWS, dtype=torch.int32), dlogprob=torch.zeros(ROWS), dentropy=None, dtotal=None)
    a.update({"strided": dict(x=wide[:, :WIDTH]), "width": dict(x=wide), "type": dict(x=x.bfloat16()), "rows": dict(residual=torch.zeros(ROWS + 1, WIDTH)),
              "tokens64": dict(tokens=torch.zeros(ROWS, dtype=torch.int64)), "dlogprob_rows": dict(dlogprob=torch.zeros(ROWS + 1)),
              "dentropy_type": dict(dentropy=torch.zeros(ROWS, dtype=torch.float64)), "dtotal_strided": dict(dtotal=wide[:, ::2])}[bad])
    with pytest.raises(ValueError):
        head.step(**a)
    if bad in ("strided", "width", "type", "rows"):
        with pytest.raises(ValueError):
            head.packed(a["x"], a["residual"])
        with pytest.raises(ValueError):
            head.score(a["x"], a["residual"], a["tokens"])


def held_bytes(head):
    """Bytes of every tensor storage that the object holds beside its parameters, states and gradients."""
    seen, todo = {}, [v for k, v in vars(head).items() if k not in ("params", "grads", "w_lowp", "m", "v", "m_scale", "v_scale", "_adam")]
    while todo:
        o = todo.pop()
        if isinstance(o, torch.Tensor):
            seen[o.untyped_storage().data_ptr()] = o.untyped_storage().nbytes()
        elif isinstance(o, dict):
            todo += o.values()
        elif isinstance(o, (list, tuple)):
            todo += o
    return sum(seen.values())


def test_ragged_calls_hold_what_the_largest_needs():
    """Every number of rows in turn, with and without alternatives, for training too: one room for the largest (logits and their gradient above all) and a few calls' results."""
    width, vocab, most = 32, 1000, 150
    head = TokenHeadStep(width, vocab, lc.LC_F32, device="cpu")
    for rows in list(range(1, most + 1)) + list(range(most, 0, -7)):
        for top in (0, 1, 20):
            head._buffers(rows, top)
        head._buffers(rows, 0, training=True)
    room = most * 4 * (2 * head.padded + 3 * width + 2) + 4 * lc.rmsnorm_bwd_workspace_bytes(lc.RmsNormDesc(most, width)) + (1 << 20)
    assert held_bytes(head) < room + 9 * most * 4 * (2 + 40 + width)


def test_results_of_another_number_of_rows_stay():
    head = TokenHeadStep(16, 40, lc.LC_F32, device="cpu")
    a, b = head._buffers(8, 0), head._buffers(3, 5)
    assert a["logprob"].data_ptr() != b["logprob"].data_ptr() and a["logits"].data_ptr() == b["logits"].data_ptr()
    assert head._buffers(8, 0) is a and head._buffers(3, 5) is b and tuple(b["logits"].shape) == (3, 40) and tuple(b["ids"].shape) == (3, 5)
    c = head._buffers(9, 0, training=True)                     # the room grows
    assert head._buffers(9, 0, training=True) is c and not c["dlogits"].any() and c["room"]["rows"] == 9


@pytest.mark.parametrize("name", ["x", "residual", "tokens", "dlogprob", "dentropy", "dtotal", "grad_scale"])
def test_tensors_of_another_device(name):
    """Checked before any launch, and without a GPU: another device than the parameters'."""
    head = TokenHeadStep(WIDTH, 40, lc.LC_F32, device="cpu")
    x, row = torch.zeros(ROWS, WIDTH), torch.zeros(ROWS)
    a = dict(x=x, residual=x, tokens=row.int(), dlogprob=row, dentropy=row, dtotal=x, grad_scale=torch.ones(1))
    a[name] = a[name].to("meta")
    with pytest.raises(ValueError, match=name):
        head.step(**a)
    if name in ("x", "residual"):
        with pytest.raises(ValueError, match=name):
            head.packed(a["x"], a["residual"])
    if name in ("x", "residual", "tokens"):
        with pytest.raises(ValueError, match=name):
            head.score(a["x"], a["residual"], a["tokens"])


@pytest.mark.parametrize("bad", [0.37, 1, torch.ones(2), torch.ones(1, dtype=torch.float64), torch.ones(1, dtype=torch.bfloat16)])
def test_gradient_scales_that_are_not_one_float_on_the_device(bad):
    head = TokenHeadStep(WIDTH, 40, lc.LC_F32, device="cpu")
    x = torch.zeros(ROWS, WIDTH)
    with pytest.raises(ValueError, match="grad_scale"):
        head.step(x, x, torch.zeros(ROWS, dtype=torch.int32), torch.zeros(ROWS), grad_scale=bad)


@pytest.mark.parametrize("residual", [True, False])
def test_no_rows(residual):
    """An empty batch is scored and packed without a launch."""
    head = TokenHeadStep(WIDTH, 40, lc.LC_F32, device="cpu")
    x, tokens = torch.zeros(0, WIDTH), torch.zeros(0, dtype=torch.int32)
    lp, ent, ids, top = head.score(x, x if residual else None, tokens, top=3)
    assert lp.shape == ent.shape == (0,) and ids.shape == top.shape == (0, 3)
    total, codes, scales = head.packed(x, x if residual else None, group=0)
    assert codes.shape == (0, WIDTH) and scales.shape == (0, 1) and (total is None) == (not residual)
