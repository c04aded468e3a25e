"""The dense head's definitions in 64 bits: the generator against published values, the
gradients against autograd and against differences."""

import math

import numpy as np
import pytest
import torch

import head_oracle as O


def test_generator_against_published_blocks():
    """The test vectors published with the generator."""
    for ctr, key, want in [
            ([0] * 4, [0] * 2, [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]),
            ([0xffffffff] * 4, [0xffffffff] * 2, [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]),
            ([0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344], [0xa4093822, 0x299f31d0],
             [0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1])]:
        got = O.philox4x32([[c] for c in ctr], key)
        assert [int(v) for v in got[:, 0]] == want


def test_kept_words_and_rate():
    w = O.philox4x32([[5], [9], [7], [1]], [3, 2])[:, 0]
    words = [int(v) >> s & 0xFFFF for v in w for s in (0, 16)]
    for p in (0.1, 0.5, 0.9):
        assert list(O.kept(8, p, 3 + (2 << 32), 7 + (1 << 32), 9, first=40)) == [
            v >= O.threshold(p) for v in words]
    n = 1 << 20
    for p in (0.1, 0.5):
        rate = 1 - O.kept(n, p, 1, 2, 3).mean()
        assert abs(rate - p) < 5 * math.sqrt(p * (1 - p) / n) + 2 ** -17
    assert O.threshold(0.0) == 0 and O.threshold(1.0) == 65536 and O.threshold(2 ** -17) == 1


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
def test_dense_gradients(act):
    r = np.random.default_rng(1)
    half = lambda *s: r.standard_normal(s).astype(np.float16)
    x, w, b, res, dy = half(5, 7), half(6, 7), half(6), half(5, 6), half(5, 6)
    X, W, B, R = (O.t64(v).requires_grad_() for v in (x, w, b, res))

    def forward(X, W, B, R):
        y = O.activate(X @ W.T + B, act)
        keep = torch.from_numpy(O.kept(30, 0.3, 11, 2, 4)).view(5, 6)
        return torch.where(keep, y * float(O.factor(0.3)), 0.0) + R
    y = forward(X, W, B, R)
    y.backward(O.t64(dy))
    z = (X @ W.T + B).detach()
    d = O.Dense(x, w, b, res, act, 0.3, (11, 2), 4, z=z.numpy(), dy=dy)
    for got, want in [(d.y, y.detach()), (d.dx, X.grad), (d.dw, W.grad), (d.db, B.grad)]:
        assert (got - want).abs().max() < 1e-12
    # differences, in a direction of each argument
    for v, g in [(X, d.dx), (W, d.dw), (B, d.db)]:
        dirn = torch.from_numpy(r.standard_normal(v.shape))
        h = 1e-6
        args = lambda s: [a.detach() + (s * h * dirn if a is v else 0) for a in (X, W, B, R)]
        num = ((forward(*args(1)) - forward(*args(-1))) * O.t64(dy)).sum() / (2 * h)
        assert abs(num - (g * dirn).sum()) < 1e-6 * max(1, abs(num))


def test_logprob_gradient():
    r = np.random.default_rng(2)
    z = (2 * r.standard_normal((4, 9))).astype(np.float16)
    z[2, 3:5] = -np.inf
    tok, dl, dh = np.array([1, -1, 0, 8], np.int32), r.standard_normal(4), r.standard_normal(4)
    L = O.Logprob(z, 1.5, 3)
    Z = O.t64(z).requires_grad_()

    def value(Z):
        lp = torch.log_softmax(Z * 1.5, 1)
        h = torch.special.entr(lp.exp()).sum(1)
        at = torch.from_numpy(tok).long().clamp(min=0)[:, None]
        t = torch.where(torch.from_numpy(tok) >= 0, lp.gather(1, at)[:, 0], 0.0)
        return (t * torch.from_numpy(dl)).sum() + (h * torch.from_numpy(dh)).sum()
    g = L.grad(tok, dl, dh)
    dirn = torch.from_numpy(r.standard_normal(z.shape))
    num = (value(Z.detach() + 1e-6 * dirn) - value(Z.detach() - 1e-6 * dirn)) / 2e-6
    assert abs(num - (g * dirn).sum()) < 1e-7 * max(1, abs(num))
    assert (g[2, 3:5] == 0).all()
    assert list(L.top_id[0]) == list(np.argsort(-z[0].astype(float), kind="stable")[:3])


def test_order_of_ties_and_nan():
    z = np.array([[1, 3, 3, np.nan, -np.inf, 0.0, -0.0]], np.float16)
    assert list(O.Logprob(z, 1.0, 7).top_id[0]) == [3, 1, 2, 0, 5, 6, 4]
