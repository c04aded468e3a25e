"""Two programs of the dense head's operators that share one generator's state and one
workspace: eager steps in turn, and a captured graph of each, replayed in turn."""

import numpy as np
import pytest
import torch

import paper_1911_07384_amd as F
from gpu_util import note
from test_gpu_head import SIZES, Program

pytestmark = pytest.mark.gpu


def test_graphs_of_two_programs_with_one_state_and_one_workspace():
    a, b = Program(*SIZES[0], seed=7), Program(*SIZES[2], seed=7)
    b.rng = a.rng
    a.ws = b.ws = max(a.ws, b.ws, key=lambda t: t.numel())
    pair, want = (a, b), []
    for i in range(6):  # a step reads the state and advances it for the other
        p = pair[i % 2]
        p.step()
        torch.cuda.synchronize()
        p.check(i)
        want.append(p.results())
    assert a.rng.tolist() == [7, 6]
    graphs = []
    for p in pair:
        note("[gpu] capture of a head")
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            p.step()
        graphs.append(g)
    a.rng.copy_(F.rng_state(7, 0))
    torch.cuda.synchronize()
    for i in range(6):
        graphs[i % 2].replay()
        if i % 3 == 2:
            torch.cuda.synchronize()
        assert np.isfinite((torch.randn(1000, device="cuda") * 2).sum().item())  # eager work
        got = pair[i % 2].results()
        assert all(np.array_equal(got[k], want[i][k], equal_nan=True) for k in got), i
    assert a.rng.tolist() == [7, 6]
