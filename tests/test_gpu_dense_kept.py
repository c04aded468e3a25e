"""The values that a dense layer keeps for its backward, with their signs."""

import numpy as np
import pytest

import head_oracle as O
from test_gpu_dense import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("tokens", [16, 990])
def test_kept_values_over_all_values(act, tokens):
    """Every finite binary16 value through an identity comes back as itself: one term of a
    sum is not 0, nothing is rounded."""
    v = np.arange(0x7C00, dtype=np.uint16).view(np.float16)
    v = np.concatenate([v, -v])
    v = np.concatenate([v, np.zeros(-v.size % (64 * tokens), np.float16)]).reshape(-1, tokens, 64)
    for part in v:
        c = Case(tokens, 64, 64, act=act, bias=False, residual=False)
        c.x, c.w = part, np.eye(64, dtype=np.float16)
        y, z = c.forward()
        assert np.array_equal(z, part)
        want = O.activate(O.t64(part), act)
        err = O.Dense.EPS * want.abs()
        O.close(y, want, err + O.HALF * (want.abs() + err) + O.TINY, act)
