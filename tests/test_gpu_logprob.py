"""GPU parity of log probabilities, entropies, the most probable classes and the logits'
gradient with their definition in 64 bits.

Bounds.  A difference of logits times the scale is off by 2 roundings of float32, and in
the exponent by two more (2^-22 of it); terms past exp(-30) do not count, so a term is
off by 30 * 2^-22 of itself and the exponential's 2^-22, S alike, plus its summation (a
lane's terms one by one, n / 256 2^-24).  log S, and with it logp, is then off by
(31 + n / 1024) 2^-22 and the roundings of the result; H by as much again for T / S,
whose terms are weighted with up to 30.  A gradient's p is off by as much relative to it,
and each rounding to binary16 by half its step."""

import numpy as np
import pytest
import torch

import head_oracle as O
import paper_1911_07384_amd as F
from gpu_util import dev, host, note, require_gpu

pytestmark = pytest.mark.gpu


def logits(rows, k, seed, spread=3.0):
    return (spread * np.random.default_rng(seed).standard_normal((rows, k))).astype(np.float16)


def given(rows, k, seed):
    t = np.random.default_rng(seed).integers(0, k, rows).astype(np.int32)
    if rows > 4:
        t[1], t[3] = -1, k  # asks for nothing; past the classes
    return t


def run(z, tokens, scale=1.0, top=0, pad=0, dlogp=None, dentropy=None, inplace=False):
    """Outputs as numpy: logp, stats, top_id, top_logp, dz (or None)."""
    require_gpu()
    rows, k = z.shape
    Z = torch.full((rows, k + pad), float("nan"), dtype=torch.float16, device="cuda")
    Z[:, :k] = dev(z)
    T = None if tokens is None else torch.from_numpy(tokens).cuda()
    d = F.logprob_desc(rows, k, stride=k + pad, scale=scale, top=top)
    f32 = dict(dtype=torch.float32, device="cuda")
    lp = torch.full((rows,), 77.0, **f32) if tokens is not None else None
    st = torch.full((rows, 3), 77.0, **f32)
    ti = torch.full((rows, top), -7, dtype=torch.int32, device="cuda") if top else None
    tl = torch.full((rows, top), 77.0, **f32) if top else None
    note(f"[gpu] logprob {rows}x{k} pad={pad} top={top} scale={scale}")
    F.fp16_logprobs(d, Z, T, lp, st, ti, tl, ws=F.workspace(F.fp16_logprobs_workspace_bytes(d)))
    torch.cuda.synchronize()
    dz = None
    if dlogp is not None or dentropy is not None:
        G = Z if inplace else torch.full_like(Z, 3.0)
        f = lambda a: None if a is None else torch.from_numpy(a.astype(np.float32)).cuda()
        note("[gpu] .. backward")
        F.fp16_logprobs_bwd(d, Z, T, st, f(dlogp), f(dentropy), G)
        torch.cuda.synchronize()
        if not inplace:
            assert bool((G[:, k:] == 3.0).all())  # the padding stays as it was
        dz = host(G[:, :k].contiguous())
    n = lambda t: None if t is None else host(t)
    return n(lp), n(st), n(ti), n(tl), dz


def check(z, tokens, scale=1.0, top=0, pad=0, dlogp=None, dentropy=None, inplace=False):
    L = O.Logprob(z, scale, top)
    lp, st, ti, tl, dz = run(z, tokens, scale, top, pad, dlogp, dentropy, inplace)
    rows, k = z.shape
    eps = (31 + k / 1024) * 2.0 ** -22
    near = lambda want: eps + 2.0 ** -22 * want.abs()
    if tokens is not None:
        t = torch.from_numpy(tokens).long()
        want = L.lp.gather(1, t.clamp(0, k - 1)[:, None])[:, 0]
        want = torch.where(t < 0, 0.0, torch.where(t >= k, float("nan"), want))
        O.close(lp, want, near(want), "logp")
    assert np.array_equal(st[:, 0], np.fmax.reduce(z.astype(np.float32), 1)) or np.isnan(z).any()
    log = torch.where(L.none, -float("inf"), L.log)
    O.close(st[:, 1], log, near(log), "log of the sum")
    O.close(st[:, 2], L.h, 31 * near(L.h), "entropy")
    if top:
        assert np.array_equal(ti, L.top_id)
        want = L.lp.gather(1, torch.from_numpy(L.top_id).long())
        O.close(tl, want, near(want), "top_logp")
    if dz is not None:
        g = L.grad(np.where(tokens is None, -1, tokens).astype(np.int32) if tokens is not None
                   else np.full(rows, -1, np.int32), dlogp, dentropy)
        dl = np.zeros(rows) if dlogp is None else dlogp
        dh = np.zeros(rows) if dentropy is None else dentropy
        lpf = torch.where(L.p > 0, L.lp, torch.zeros_like(L.lp))
        mag = torch.from_numpy(np.abs(dl))[:, None] + torch.from_numpy(np.abs(dh))[:, None] * (
            lpf.abs() + L.h.abs()[:, None] + 1)
        # p and log p + H by their bounds, the sum of both terms by float32 roundings
        err = 40 * eps * L.s * mag * L.p + 8 * O.F32 * L.s * (
            mag * L.p + torch.from_numpy(np.abs(dl))[:, None])
        err = torch.nan_to_num(err, nan=0.0)
        O.close(dz, g, err + O.HALF * (g.abs() + err) + O.TINY, "dz")


SIZES = [(1, 1), (1, 2), (3, 5), (2, 8), (5, 64), (7, 100), (4, 1000), (128, 1000), (33, 1025),
         (2, 2047), (3, 4097), (600, 333), (1, 8193), (1, 131071), (2, 50001), (700, 8200)]


@pytest.mark.parametrize("size", SIZES, ids=lambda s: f"{s[0]}x{s[1]}")
def test_values_and_gradients(size):
    rows, k = size
    r = np.random.default_rng(rows + k)
    z = logits(rows, k, rows * 7 + k)
    check(z, given(rows, k, 3), 1.0, min(5, k), 0, r.standard_normal(rows),
          0.1 * r.standard_normal(rows))


@pytest.mark.parametrize("top", [1, 2, 20, 63, 64])
@pytest.mark.parametrize("size", [(5, 64), (3, 1000), (2, 5000), (1, 70001), (520, 4300)],
                         ids=lambda s: f"{s[0]}x{s[1]}")
def test_most_probable(size, top):
    check(logits(*size, top), given(*size, 1), 0.7, top)


@pytest.mark.parametrize("pad", [1, 3, 8, 47])
def test_strides(pad):
    for rows, k in [(9, 1001), (3, 9000), (700, 77)]:
        check(logits(rows, k, pad), given(rows, k, pad), 1.3, 4, pad, np.ones(rows), np.ones(rows))


@pytest.mark.parametrize("size", [(3, 64), (2, 3000), (1, 40000), (513, 9000)],
                         ids=lambda s: f"{s[0]}x{s[1]}")
def test_equal_logits(size):
    """More equal values than any buffer of candidates holds; the lower classes win."""
    rows, k = size
    for z in (np.zeros(size), np.random.default_rng(k).integers(-1, 2, size),
              np.where(np.arange(k) == k - 1, 2.0, -1.5)[None].repeat(rows, 0)):
        check(z.astype(np.float16), given(rows, k, 2), 1.0, 64, 1, np.ones(rows), np.ones(rows))


def test_sorted_rows():
    k = 20000
    up = np.linspace(-20, 20, k).astype(np.float16)
    check(np.stack([up, up[::-1]]), np.array([k - 1, 0], np.int32), 1.0, 64)


@pytest.mark.parametrize("k", [7, 600, 9001, 40000])
def test_masked_classes(k):
    """-inf in single places, whole runs, everything but one class, and everything."""
    z = logits(6, k, k)
    z[0, ::3] = -np.inf
    z[1, k // 2:] = -np.inf
    z[2] = -np.inf
    z[2, k - 1] = -3.0
    z[3] = -np.inf
    z[4, :k - 1] = -65504.0  # the type's lowest value as a mask
    tokens = np.array([0, k - 1, k - 1, 1, k - 1, 2], np.int32)
    r = np.random.default_rng(k)
    check(z, tokens, 1.0, min(k, 9), 0, r.standard_normal(6), r.standard_normal(6))


@pytest.mark.parametrize("k", [5, 700, 9001])
def test_values_that_are_not_finite(k):
    z = logits(5, k, k)
    z[0, k // 2] = np.nan
    z[1, 1] = np.inf
    z[2, k - 1], z[2, 0] = np.nan, np.inf
    z[3] = np.nan
    L = O.Logprob(z, 1.0, 3)
    lp, st, ti, tl, dz = run(z, np.array([0, 1, 2, 3, 4], np.int32), 1.0, 3, 0, np.ones(5),
                             np.ones(5))
    assert np.isnan(lp[:4]).all() and np.isnan(st[:4, 2]).all() and np.isnan(tl[:4]).all()
    assert np.isnan(dz[:4]).all() and np.isfinite(dz[4]).all() and np.isfinite(lp[4])
    assert np.array_equal(ti, L.top_id)


def test_sizes_of_logits_and_scales():
    """Logits at the ends of the type and scales far from 1: the differences count."""
    r = np.random.default_rng(5)
    z = (65504 - 32.0 * r.integers(0, 40, (4, 3001))).astype(np.float16)
    check(z, given(4, 3001, 1)[:4] % 3001, 0.05, 5, 0, np.ones(4), np.ones(4))
    check(-z, given(4, 3001, 1)[:4] % 3001, 0.05, 5, 0, np.ones(4), np.ones(4))
    z = logits(4, 3001, 9, spread=2.0 ** -12)
    check(z, given(4, 3001, 1)[:4] % 3001, 1000.0, 5, 0, np.ones(4), np.ones(4))
    check(logits(4, 300, 8), given(4, 300, 1), 1e-6, 5, 0, np.ones(4), np.ones(4))
    check(logits(4, 300, 8), given(4, 300, 1)[:4], 500.0, 5, 0, np.ones(4), np.ones(4))


def test_parts_of_the_outputs():
    z, t = logits(6, 2500, 1), given(6, 2500, 4)
    check(z, None, 1.0, 3)
    check(z, None, 1.0, 0, 0, None, np.ones(6))
    check(z, t, 1.0, 0, 0, np.ones(6), None)
    check(z, t, 1.0, 0, 2, np.ones(6), np.ones(6), inplace=True)


def test_gradient_against_differences():
    """The change of the outputs along a direction, from the kernels' own values."""
    rows, k = 3, 40
    z = np.round(logits(rows, k, 2) * 64).astype(np.float16) / np.float16(64)
    t = np.array([3, 39, 0], np.int32)
    dl, dh = np.array([1.0, -2.0, 0.5]), np.array([0.3, 1.0, -1.0])
    *_, dz = run(z, t, 1.0, 0, 0, dl, dh)
    h = np.float16(2.0 ** -5)
    dirn = np.random.default_rng(1).integers(-1, 2, z.shape).astype(np.float16)
    out = []
    for s in (1, -1):
        lp, st, *_ = run((z + s * h * dirn).astype(np.float16), t)
        out.append((lp.astype(np.float64) * dl).sum() + (st[:, 2].astype(np.float64) * dh).sum())
    num = (out[0] - out[1]) / (2 * float(h))
    # h^2 of third derivatives below 6 (3.5) x 3 rows, roundings of the values over 2h
    assert abs(num - (dz.astype(np.float64) * dirn).sum()) < 18 * 2.0 ** -10 + 1e-3


def test_large_gradients_of_masked_classes():
    z = logits(3, 700, 4)
    z[:, 5:300] = -np.inf
    z[2, 400:] = -65504  # (a probability of 0, but for the scale)
    dz = run(z, None, scale=4.0, dentropy=np.full(3, 1e32))[-1]
    assert (dz[:, 5:300] == 0).all() and (dz[2, 400:] == 0).all() and not np.isnan(dz).any()


def test_same_bits_every_time():
    z, t = logits(40, 20011, 3), given(40, 20011, 5)
    z[5] = 1.0
    a = run(z, t, 1.0, 20, 1, np.ones(40), np.ones(40))
    for _ in range(3):
        b = run(z, t, 1.0, 20, 1, np.ones(40), np.ones(40))
        assert all(np.array_equal(p, q, equal_nan=True) for p, q in zip(a, b))


@pytest.mark.parametrize("top", [0, 20, 64])
def test_many_long_rows(top):
    """Whole rows of a wider workgroup's own."""
    for k in (16385, 17003):
        r = np.random.default_rng(k)
        check(logits(512, k, k), given(512, k, 1), 0.9, top, 5, r.standard_normal(512),
              r.standard_normal(512))
        z = np.zeros((512, k))
        z[:256, ::3] = -np.inf
        check(z.astype(np.float16), given(512, k, 2), 1.0, top)
