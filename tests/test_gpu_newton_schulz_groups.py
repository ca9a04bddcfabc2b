"""Lists of more matrices than a launch takes: each group of them goes by the kernels that its own sizes ask for, whatever other groups hold."""
import ctypes

import numpy as np
import pytest
import torch

from paper_1709_05011_amd import larsconv as lc
from paper_1709_05011_amd import synth

import gpu_util as gu
from test_gpu_newton_schulz import check_step

pytestmark = pytest.mark.gpu


def launches_of(call):
    """Kernels that a graph records of a call."""
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph):
        call()
    count = ctypes.c_size_t()
    get = lc.lib().hipGraphGetNodes
    get.restype, get.argtypes = ctypes.c_int, [ctypes.c_void_p, ctypes.c_void_p, ctypes.POINTER(ctypes.c_size_t)]
    assert get(ctypes.c_void_p(graph.raw_cuda_graph()), None, ctypes.byref(count)) == 0
    return count.value


def test_one_large_matrix_among_many_small_ones():
    """330 x 350 goes with the 63 longest of 150 small matrices through a launch a product; the other 87 take one launch for each group of 64.  Updates against 64 bits."""
    shapes = [(5 + i % 60, 3 + (i * 7) % 250) for i in range(150)]
    shapes.insert(70, (330, 350))
    w, g, m = ([gu.dev(synth.normal(s, k + 5 * i, std=std)) for i, s in enumerate(shapes)] for k, std in ((0, 0.02), (1, 1e-3), (2, 4e-3)))
    before = [[t.clone() for t in v] for v in (w, g, m)]
    args = lc.MuonArgs(w, g, m)
    ws = gu.workspace(lc.muon_workspace_bytes(args))
    step = lambda a: lc.muon_step(a, 0.02, 0.95, 0.1, ws)
    step(args)
    torch.cuda.synchronize()
    check_step(shapes, before, (w, m), None, 0.02, 0.95, float(np.float32(0.1)), True, None)
    one = lc.MuonArgs(w[70:71], g[70:71], m[70:71])
    small = [v[:70] + v[71:134] for v in (w, g, m)]                # 133 small ones: three groups
    torch.cuda.synchronize()
    alone, few, all_of_them = launches_of(lambda: step(one)), launches_of(lambda: step(lc.MuonArgs(*small))), launches_of(lambda: step(args))
    assert alone > 3 and few == 3
    assert all_of_them == alone + 2                                # 151 matrices: the first group as the large one by itself, two of small ones
