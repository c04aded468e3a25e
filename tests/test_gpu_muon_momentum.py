"""The momentum of fp16_muon_step on both of its paths (one workgroup a matrix; tiles
over all CUs): without Nesterov's look-ahead, and with one whose squares pass float32."""

import numpy as np
import pytest
import torch

import oracle
import paper_1911_07384_amd as F
from gpu_util import host, note, require_gpu
from test_gpu_muon import BAR, matrix, ns64, off, step

pytestmark = pytest.mark.gpu

SETS = {"workgroup": [(64, 147), (147, 64), (5, 3), (33, 1000), (1000, 33), (1, 9)],
        "tiles": [(65, 147), (147, 65), (5, 3), (33, 1030), (1030, 33), (1, 9)]}


def paths(shapes):
    return F.fp16_muon_kernels(F.muon_descs(shapes), 1) == "one workgroup each"


@pytest.mark.parametrize("products", [1, 3])
@pytest.mark.parametrize("path", SETS)
def test_plain_momentum(path, products):
    """nesterov = 0: the direction is the rounded momentum alone.  Weights from zero
    without decay, so that they hold the direction to its bar and one rounding."""
    require_gpu()
    shapes = SETS[path]
    assert paths(shapes) == (path == "workgroup")
    g = [matrix(*s, seed=10 + i) for i, s in enumerate(shapes)]
    m = [matrix(*s, seed=20 + i) for i, s in enumerate(shapes)]
    W = [torch.zeros(s, dtype=torch.float16, device="cuda") for s in shapes]
    G, M = ([t.cuda() for t in l] for l in (g, m))
    step(W, G, M, [1.0] * len(shapes), 0.5, 0.95, 0.0, False, products)
    for i, s in enumerate(shapes):
        _, mr = oracle.sgd_f32(np.zeros(g[i].numel(), np.float16), g[i].numpy().ravel(),
                               m[i].numpy().ravel(), 0.1, 0.95, 0.0)
        assert np.array_equal(host(M[i]).ravel().view(np.uint16), mr.view(np.uint16))
        ref = -0.5 * ns64(torch.from_numpy(mr).view(*s))
        assert off(W[i], ref) <= BAR[products], s
        assert torch.equal(G[i].cpu(), g[i])


@pytest.mark.parametrize("path", SETS)
def test_momentum_whose_squares_pass_float32(path):
    """From a zero momentum the direction is (mu + 1) g whatever mu: with mu = 2^80
    its squares, about 2^138, are finite in float64 only."""
    require_gpu()
    shapes = SETS[path]
    g = [matrix(*s, seed=30 + i) for i, s in enumerate(shapes)]
    W, M = ([torch.zeros(s, dtype=torch.float16, device="cuda") for s in shapes] for _ in range(2))
    note("[gpu] a momentum of 2^80")
    step(W, [t.cuda() for t in g], M, [1.0] * len(shapes), 0.5, 2.0 ** 80, 0.0, True, 3)
    for i, s in enumerate(shapes):
        assert torch.equal(M[i].cpu(), g[i])
        assert off(W[i], -0.5 * ns64(g[i])) <= BAR[3], s
