"""GPU parity of the counter-based dropout: every result is one bit pattern."""

import numpy as np
import pytest
import torch

import head_oracle as O
import paper_1911_07384_amd as F
from gpu_util import dev, host, note, require_gpu

pytestmark = pytest.mark.gpu


def values(n, seed):
    return np.random.default_rng(seed).standard_normal(n).astype(np.float16)


def same(a, b):
    na, nb = np.isnan(a), np.isnan(b)
    return np.array_equal(na, nb) and np.array_equal(a[~na].view(np.uint16), b[~nb].view(np.uint16))


def run(x, res, p, seed=5, step=3, site=2, inplace=None):
    require_gpu()
    X, R = dev(x), None if res is None else dev(res)
    n = x.size
    pad = torch.full((n + 64,), 7.0, dtype=torch.float16, device="cuda")
    Y = {None: pad[:n], "x": X, "residual": R}[inplace]
    note(f"[gpu] dropout n={n} p={p} residual={res is not None} in place: {inplace}")
    F.fp16_dropout(X, R, Y, p, F.rng_state(seed, step), site=site)
    torch.cuda.synchronize()
    assert bool((pad[n:] == 7.0).all())  # nothing behind the end
    return host(Y)


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("n", [1, 7, 8, 9, 255, 2048, 2055, 16384 + 5, 1 << 20, 3_000_001])
def test_values(n, residual):
    x = values(n, n)
    res = values(n, n + 1) if residual else None
    for p in (0.1, 0.5):
        assert same(run(x, res, p), O.dropout(x, res, p, 5, 3, 2))


@pytest.mark.parametrize("p", [0.0, 2.0 ** -18, 2.0 ** -17, 2.0 ** -16, 0.3333, 0.999, 1.0 - 2 ** -16,
                               1.0])
def test_probabilities(p):
    x, res = values(70001, 1), values(70001, 2)
    assert same(run(x, res, p), O.dropout(x, res, p, 5, 3, 2))
    assert same(run(x, None, p), O.dropout(x, None, p, 5, 3, 2))


@pytest.mark.parametrize("seed,step,site", [(0, 0, 0), (2 ** 64 - 1, 2 ** 64 - 1, 2 ** 32 - 1),
                                            (1 << 40, 3, 0), (3, 1 << 40, 7), (3, 0, 1 << 31)])
def test_states(seed, step, site):
    x = values(5003, 4)
    assert same(run(x, None, 0.25, seed, step, site), O.dropout(x, None, 0.25, seed, step, site))


@pytest.mark.parametrize("inplace", ["x", "residual"])
def test_in_place(inplace):
    x, res = values(12345, 5), values(12345, 6)
    assert same(run(x, res, 0.3, inplace=inplace), O.dropout(x, res, 0.3, 5, 3, 2))


def test_dropped_values_are_not_looked_at():
    x, res = values(4096, 7), values(4096, 8)
    keep = O.kept(4096, 0.5, 5, 3, 2)
    x[~keep] = np.tile(np.array([np.nan, np.inf, -np.inf], np.float16), 4096)[:(~keep).sum()]
    y = run(x, res, 0.5)
    assert np.isfinite(y).all() and same(y[~keep], res[~keep] + np.float16(0))
    x = np.where(keep, np.float16(np.nan), x)
    assert np.isnan(run(x, res, 0.5)[keep]).all()


def test_overflow_and_subnormals():
    x = np.concatenate([np.full(512, 60000, np.float16), np.full(512, 2.0 ** -24, np.float16),
                        np.full(512, -0.0, np.float16)])
    for p in (0.1, 0.5):
        assert same(run(x, None, p), O.dropout(x, None, p, 5, 3, 2))


def test_more_elements_than_32_bits_hold():
    """The last elements of 2^32 + 4091."""
    require_gpu()
    n, tail = (1 << 32) + 4091, 8192
    x = torch.ones(n, dtype=torch.float16, device="cuda")
    y = torch.empty_like(x)
    note(f"[gpu] dropout n={n}")
    F.fp16_dropout(x, None, y, 0.4, F.rng_state(9, 1), site=5)
    torch.cuda.synchronize()
    first = n // 8 * 8 - tail
    want = np.where(O.kept(n - first, 0.4, 9, 1, 5, first=first), O.factor(0.4), 0)
    assert same(host(y[first:]), want.astype(np.float16))


def test_advance():
    require_gpu()
    s = F.rng_state(77, (1 << 32) - 1)
    F.fp16_rng_advance(s)
    F.fp16_rng_advance(s, 1 << 33)
    assert s.tolist() == [77, (1 << 32) + (1 << 33)]
    s = F.rng_state(1, 2 ** 64 - 1)
    F.fp16_rng_advance(s, 2)
    assert s.tolist() == [1, 1]
