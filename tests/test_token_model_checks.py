"""A token model's step refuses tensors that the entry points' pointers would misread, before any launch (no GPU needed)."""
import pytest
import torch

from paper_1709_05011_amd import larsconv as lc
from paper_1709_05011_amd.token_model_step import TokenModelStep

ROWS = 4


@pytest.mark.parametrize("bad", ["tokens64", "tokens_rows", "tokens_strided", "targets_none", "targets_float", "dlogprob_rows", "dlogprob_none", "dentropy_type", "grad_scale", "grad_scale_float"])
def test_refusals(bad):
    model = TokenModelStep(16, 40, 2, lc.LC_F32, device="cpu")
    i32 = lambda n: torch.zeros(n, dtype=torch.int32)
    a = dict(tokens=i32(ROWS), targets=i32(ROWS), dlogprob=torch.zeros(ROWS), dentropy=None, grad_scale=None)
    a.update({"tokens64": dict(tokens=torch.zeros(ROWS, dtype=torch.int64)), "tokens_rows": dict(tokens=i32(ROWS + 1)), "tokens_strided": dict(tokens=i32(2 * ROWS)[::2]),
              "targets_none": dict(targets=None), "targets_float": dict(targets=torch.zeros(ROWS)), "dlogprob_rows": dict(dlogprob=torch.zeros(ROWS + 1)),
              "dlogprob_none": dict(dlogprob=None), "dentropy_type": dict(dentropy=torch.zeros(ROWS, dtype=torch.float64)), "grad_scale": dict(grad_scale=torch.zeros(2)),
              "grad_scale_float": dict(grad_scale=0.5)}[bad])
    with pytest.raises(ValueError):
        model.step(**a)
    if bad.startswith(("tokens", "targets")):
        with pytest.raises(ValueError):
            model.score(a["tokens"], a["targets"])
    assert model.steps == 0
