"""Log probabilities, entropies, the most probable classes and the logits' gradient at
every size of the scale, against their definition in 64 bits, with the bounds of
test_gpu_logprob: a difference of two logits times the scale is off by 2^-22 of itself
whatever the logits' size.  The gradients of logp and of the entropy are taken over the
scale, so that the logits' are of the size of 1 at every scale."""

import numpy as np
import pytest

import head_oracle as O
from test_gpu_logprob import check, given, logits, run

pytestmark = pytest.mark.gpu

# both sides of where a product of a logit and the scale needs more bits than a float32
# has for its whole part (about 177), and the ends of the declared range
SCALES = [1e-40, 1e-6, 170.0, 177.0, 178.0, 500.0, 3e4, 1e5, 1e6, 1e9, 1e12, 1e30]


def rows_of(k, scale, seed):
    """Ordinary logits; lanes of nothing but a finite mask; the type's ends; equal ones; steps of
    the smallest subnormal; masked ones; all masked."""
    r = np.random.default_rng(seed)
    z = logits(12, k, seed)
    z[1, k // 3:] = -65504.0
    z[2] = -65504.0
    z[2, k // 2] = 7.1
    z[3] = (65504 - 32.0 * r.integers(0, 40, k)).astype(np.float16)
    z[4] = -z[3]
    z[5] = -65504.0
    z[6] = 11.3
    z[7] = (r.integers(-1000, 1000, k) * 2.0 ** -24).astype(np.float16)
    z[8, ::2] = -np.inf
    z[9] = -np.inf
    z[10] = np.float16(60000.0) * np.sign(logits(1, k, seed + 1))[0]
    z[11] = -np.inf
    z[11, k - 1] = 3.7
    return z


def both(z, scale, top, pad, seed):
    rows, k = z.shape
    r = np.random.default_rng(seed)
    over = max(scale, 1e-6)
    check(z, given(rows, k, seed), scale, min(top, k), pad, r.standard_normal(rows) / over,
          0.1 * r.standard_normal(rows) / over)


@pytest.mark.parametrize("scale", SCALES)
@pytest.mark.parametrize("k", [3, 700, 2500, 9001])
def test_scales(k, scale):
    """Rows of one workgroup and (9001) in parts."""
    both(rows_of(k, scale, k), scale, 20, 3, k)


@pytest.mark.parametrize("scale", [170.0, 3e4, 1e9, 1e30])
def test_scales_of_long_rows(scale):
    """Rows in many parts, and many rows of a wide workgroup's own."""
    both(rows_of(60001, scale, 1), scale, 64, 0, 2)
    z = np.tile(rows_of(16390, scale, 3), (43, 1))
    both(z, scale, 20, 0, 4)


@pytest.mark.parametrize("scale", [1e5, 1e9, 1e30])
@pytest.mark.parametrize("top", [0, 3])
def test_equal_largest_logits(top, scale):
    """Entropies log 2 and log 3, and gradients that cancel to nothing between them."""
    z = logits(4, 1000, 5)
    z[0, [3, 700]] = 40.3
    z[1, [0, 500, 999]] = 12345.0
    z[2, 17:19] = -0.001
    z[2, :17], z[2, 19:] = -50.0, -60.0
    z[3, 8:] = -65504.0
    z[3, [1, 2]] = 31.7
    check(z, np.array([3, 1, 18, 2], np.int32), scale, top, 0, np.ones(4) / scale,
          np.ones(4) / scale)
    *_, dz = run(z, None, scale, 0, 0, None, np.ones(4))
    assert (dz == 0).all()


@pytest.mark.parametrize("k", [5, 700, 9001])
@pytest.mark.parametrize("scale", [3e4, 1e9])
def test_values_that_are_not_finite(k, scale):
    z = logits(5, k, k)
    z[0, k // 2] = np.nan
    z[1, 1] = np.inf
    z[2, k - 1], z[2, 0] = np.nan, np.inf
    z[3] = np.nan
    L = O.Logprob(z, scale, 3)
    lp, st, ti, tl, dz = run(z, np.array([0, 1, 2, 3, 4], np.int32), scale, 3, 0, np.ones(5) / scale,
                             np.ones(5) / scale)
    assert np.isnan(lp[:4]).all() and np.isnan(st[:4, 1:]).all() and np.isnan(tl[:4]).all()
    assert np.isnan(dz[:4]).all() and np.isfinite(dz[4]).all() and np.isfinite(lp[4])
    assert np.array_equal(ti, L.top_id)
