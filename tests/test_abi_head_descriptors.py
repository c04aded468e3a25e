"""Descriptors of the dense head: a number that its field does not hold is refused, and
not cut to another one."""

import pytest

import paper_1911_07384_amd as F

A, B, R = 0x1000000000, 0x2000000000, 0x3000000000


@pytest.mark.parametrize("big", [1 << 31, (1 << 32) + 5, 1 << 40, -(1 << 31) - 1])
def test_sizes_past_32_bits(big):
    for k in ("tokens", "inputs", "outputs"):
        with pytest.raises(ValueError, match=k):
            F.dense_desc(**{"tokens": 4, "inputs": 8, "outputs": 16, k: big})
    for k in ("rows", "classes", "stride", "top"):
        with pytest.raises(ValueError, match=k):
            F.logprob_desc(**{"rows": 4, "classes": 8, "stride": 16, k: big})
    with pytest.raises(ValueError, match="act"):
        F.dense_desc(4, 8, 16, act=big)


@pytest.mark.parametrize("site", [1 << 32, (1 << 32) + 3, -1, 1 << 64])
def test_sites_past_32_bits(site):
    with pytest.raises(ValueError, match="site"):
        F.dense_desc(4, 8, 16, drop=0.5, site=site)
    with pytest.raises(ValueError, match="site"):
        F.fp16_dropout(A, None, B, 0.5, R, site=site, n=0, stream=0)


def test_the_largest_numbers_are_taken():
    m = (1 << 31) - 1
    d = F.dense_desc(m, m, m, site=(1 << 32) - 1)
    assert (d.tokens, d.inputs, d.outputs, d.site) == (m, m, m, (1 << 32) - 1)
    assert F.logprob_desc(m, -m - 1, stride=m).classes == -m - 1
    F.fp16_dropout(A, None, B, 0.5, R, site=(1 << 32) - 1, n=0, stream=0)
