"""The logits' gradient where the gradient of the entropy is as large as a float32 gets."""

import numpy as np
import pytest
import torch

import head_oracle as O
from test_gpu_logprob import logits, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dentropy", [1e32, 1e36, 1e37, 3e38, -3e38])
def test_classes_of_probability_0(dentropy):
    """Masked by -inf or by the type's lowest value: 0, whatever the entropy's gradient."""
    z = logits(3, 700, 4)
    z[:, 5:300] = -np.inf
    z[2, 400:] = -65504
    for dlogp in (None, np.ones(3)):
        tokens = None if dlogp is None else np.array([0, 1, 2], np.int32)
        dz = run(z, tokens, scale=4.0, dlogp=dlogp, dentropy=np.full(3, dentropy))[-1]
        assert (dz[:, 5:300] == 0).all() and (dz[2, 400:] == 0).all() and not np.isnan(dz).any()


@pytest.mark.parametrize("dentropy", [1e36, 1e37, 1e38])
def test_small_probabilities(dentropy):
    """p of some 1e-36 times an entropy's gradient of 1e37: the product is of the size of 1.

    log p is off by 2^-23 of itself and 2^-24 of the log of the sum, its product with 1 / ln 2 by 2^-23
    more (the constant's rounding and its own), so p by 86 * 2^-22 and an exponential's 2^-22 of itself;
    log p + H, of some -80, by 2^-22 of itself, the three products by 2^-24 each, and the result by
    half its step."""
    z = np.full((2, 64), -86.0, np.float16)
    z[:, 3] = 0.0
    z[:, 10:20] = -83.0 + np.arange(10) * 0.0625
    dz = run(z, None, dentropy=np.full(2, dentropy))[-1]
    L = O.Logprob(z)
    want = L.grad(np.full(2, -1, np.int32), None, np.full(2, float(np.float32(dentropy))))
    small = L.p < 0.5
    err = (90 * 2.0 ** -22 + O.HALF) * want.abs() + O.TINY
    got = torch.from_numpy(dz).double()
    over = want.abs() >= 65504
    assert bool(((got - want).abs() <= err)[small & ~over].all())
    assert bool(torch.isinf(got)[small & (want.abs() > 65600)].all())
    assert bool((small & ~over & (want.abs() > 1e-3)).any())
