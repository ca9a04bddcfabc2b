"""Descriptors of the token operators as values: a used one is equal to, hashes, copies and travels like a fresh one (no GPU needed)."""
import copy
import dataclasses
import pickle

import pytest

from paper_1709_05011_amd import larsconv as lc


@pytest.mark.parametrize("desc,use", [(lc.RmsNormDesc(40, 100, x_ld=128, dtype=lc.LC_BF16), lc.rmsnorm_bwd_workspace_bytes),
                                      (lc.TokenDesc(4, 131072, top=5), lc.token_logprob_workspace_bytes)])
def test_a_used_descriptor_is_a_value(desc, use):
    fresh, need = dataclasses.replace(desc), use(desc)
    assert need > 0 and use(desc) == need
    for other in (pickle.loads(pickle.dumps(desc)), copy.copy(desc), copy.deepcopy(desc), dataclasses.replace(desc), fresh):
        assert other == desc and hash(other) == hash(desc) and use(other) == need and repr(other) == repr(desc)
    wider = dataclasses.replace(desc, rows=2 * desc.rows)
    assert use(wider) != need and wider != desc
