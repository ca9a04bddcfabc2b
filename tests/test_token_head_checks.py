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
