"""Definitions in 64 bits of the dense head's operators: the generator and dropout,
dense layers with their epilogue and backward, log probabilities and their gradient.
Everything is numpy or torch float64 on the CPU."""

from __future__ import annotations

import math

import numpy as np
import torch

HALF = 2.0 ** -11     # a rounding to binary16, relative
TINY = 2.0 ** -25     # .. and absolute, half its smallest step
F32 = 2.0 ** -24


def philox4x32(ctr, key, rounds=10):
    """Blocks of the generator: ctr [4][n] and key (2) of 32-bit values -> [4][n]."""
    u, low = np.uint64, np.uint64(0xFFFFFFFF)
    c = [np.array(v, dtype=np.uint64) for v in ctr]
    k = [int(v) for v in key]
    for _ in range(rounds):
        a, b = c[0] * u(0xD2511F53), c[2] * u(0xCD9E8D57)
        c = [(b >> u(32)) ^ c[1] ^ u(k[0]), b & low, (a >> u(32)) ^ c[3] ^ u(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) % 2 ** 32, (k[1] + 0xBB67AE85) % 2 ** 32]
    return np.stack(c)


def threshold(p):
    return int(math.floor(float(np.float32(p)) * 65536 + 0.5))


def kept(n, p, seed, step, site, first=0):
    """Which of the elements first .. first + n - 1 are kept (first a multiple of 8)."""
    g = np.arange(first // 8, first // 8 + -(-n // 8), dtype=np.uint64)
    one = np.ones_like(g)
    w = philox4x32([g, one * np.uint64(site), one * np.uint64(step % 2 ** 32),
                    one * np.uint64((step >> 32) % 2 ** 32)],
                   [seed % 2 ** 32, (seed >> 32) % 2 ** 32])
    words = np.stack([w & np.uint64(0xFFFF), w >> np.uint64(16)], 1)  # [4][2][groups]
    return words.reshape(8, -1).T.reshape(-1)[:n] >= threshold(p)


def factor(p):
    """What kept values are multiplied by, as the float32 that is declared."""
    t = threshold(p)
    return np.float32(65536.0 / (65536 - t)) if t < 65536 else np.float32(0.0)


def dropout(x16, residual16, p, seed, step=0, site=0):
    """The declared float32 sequence, to binary16."""
    keep = kept(x16.size, p, seed, step, site).reshape(x16.shape)
    with np.errstate(invalid="ignore", over="ignore"):
        v = np.where(keep, x16.astype(np.float32) * factor(p), np.float32(0.0))
        if residual16 is not None:
            v = v + residual16.astype(np.float32)
        return v.astype(np.float16)


def phi(z):
    return torch.special.ndtr(z)


def activate(z, act):
    if act == "relu":
        return torch.where(z > 0, z, torch.where(z.isnan(), z, 0.0))
    if act == "gelu":
        return torch.where(z < -40, 0.0, z * phi(z))
    if act == "silu":
        return torch.where(z < -700, 0.0, z * torch.sigmoid(z))
    return z


def slope(z, act):
    if act == "relu":
        return torch.where(z > 0, 1.0, torch.where(z.isnan(), z, 0.0))
    if act == "gelu":
        v = phi(z) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
        return torch.where(z.abs() > 40, (z > 0).double(), v)
    if act == "silu":
        s = torch.sigmoid(z)
        return torch.where(z.abs() > 700, (z > 0).double(), s * (1 + z * (1 - s)))
    return torch.ones_like(z)


def t64(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).double()


class Dense:
    """A layer's outputs and gradients, each with a bound on its error: float32 sums of
    n terms in any order are off by at most (n + 2) 2^-23 of the terms' magnitudes (a
    matrix core may cut a sum's last bit instead of rounding it), the activations and
    slopes by EPS of a value, each rounding to binary16 by half its step."""

    EPS = 2.0 ** -16

    def __init__(self, x, w, bias=None, residual=None, act="none", p=0.0, rng=(0, 0), site=0,
                 z=None, dy=None):
        X, W = t64(x), t64(w)
        tokens, outputs = x.shape[0], w.shape[0]
        k = x.shape[1]
        v = X @ W.T
        mag = X.abs() @ W.abs().T
        if bias is not None:
            v, mag = v + t64(bias), mag + t64(bias).abs()
        dv = (k + 2) * 2.0 ** -23 * mag
        self.v, self.z, self.z_err = v, v, dv + HALF * (v.abs() + dv) + TINY
        keep = torch.from_numpy(kept(tokens * outputs, p, rng[0], rng[1], site)
                                if threshold(p) else np.ones(tokens * outputs, bool))
        self.scale = s = float(factor(p))
        keep = self.keep = keep.view(tokens, outputs)
        a = activate(v, act)
        y = torch.where(keep, a * s, 0.0)
        # no slope is above 1.13
        err = torch.where(keep, s * (1.13 * dv + (self.EPS + 2 * F32) * a.abs()), 0.0)
        if residual is not None:
            y = y + t64(residual)
            err = err + F32 * y.abs()
        self.y, self.y_err = y, err + HALF * (y.abs() + err) + TINY
        if dy is None:
            return
        u = torch.where(keep, t64(dy) * s, 0.0)
        if act != "none":
            u = u * slope(t64(z), act)
        # (relative to dy: a slope near its zero is off by EPS of 1)
        du = (self.EPS + 4 * F32) * torch.where(keep, t64(dy).abs() * s, 0.0)
        if act == "none" and s == 1.0:
            dz_err = torch.zeros_like(u)
            du = torch.zeros_like(u)
        else:
            dz_err = du + HALF * (u.abs() + du) + TINY
        self.u = u
        um = u.abs() + dz_err

        def out(value, err, mag, n):
            e = err + (n + 2) * 2.0 ** -23 * mag
            return value, e + HALF * (value.abs() + e) + TINY
        self.dx, self.dx_err = out(u @ W, dz_err @ W.abs(), um @ W.abs(), outputs)
        self.dw, self.dw_err = out(u.T @ X, dz_err.T @ X.abs(), um.T @ X.abs(), tokens)
        self.db, self.db_err = out(u.sum(0), du.sum(0), u.abs().sum(0), tokens)


def close(got, want, err, what):
    """Every element within its bound; NaN and infinities where they belong."""
    g = torch.from_numpy(np.ascontiguousarray(got)).double()
    assert g.shape == want.shape, (what, g.shape, want.shape)
    big = want.abs() > 65504.0 - err - 16.0  # may round to infinity
    odd = ~torch.isfinite(want)
    assert torch.equal(g.isnan(), want.isnan()), what
    same = (g == want) | (want.isnan() & g.isnan())
    assert bool(same[odd].all()), what
    off = ((g - want).abs() > err) & ~odd & ~(big & (g.isinf() | (g.abs() > 60000)))
    if bool(off.any()):
        i = tuple(int(v) for v in off.nonzero()[0])
        raise AssertionError(f"{what}: {int(off.sum())} of {off.numel()} off, first at {i}: "
                             f"{g[i]} for {want[i]} within {err[i]}")


class Logprob:
    """Log probabilities in 64 bits, and each row's classes in order."""

    def __init__(self, z16, scale=1.0, top=0):
        z = t64(z16)
        s = float(np.float32(scale))
        m = z.amax(1, keepdim=True)
        self.none = (m == -math.inf)[:, 0]
        d = (z - torch.where(torch.isinf(m) & (m < 0), 0.0, m)) * s
        e = torch.exp(d)
        total = e.sum(1, keepdim=True)
        log = torch.log(total)
        self.m, self.log = m[:, 0], log[:, 0]
        self.lp = d - log
        self.lp[self.none] = -math.inf
        p = e / total
        self.h = -torch.where(p > 0, p * self.lp, torch.where(p.isnan(), p, 0.0)).sum(1)
        self.h[self.none] = 0.0
        self.p, self.s = p, s
        # NaN above everything, then the values, then the lower class (stable)
        key = np.where(np.isnan(z16), np.inf, z16.astype(np.float64))
        rows = []
        for r in range(z16.shape[0]):
            rows.append(np.lexsort((np.arange(z16.shape[1]), -key[r], ~np.isnan(z16[r])))[:top])
        self.top_id = np.array(rows, dtype=np.int32).reshape(z16.shape[0], top)

    def grad(self, tokens, dlogp, dentropy):
        n, k = self.lp.shape
        t = torch.from_numpy(tokens).long()
        dl = torch.zeros(n, dtype=torch.float64) if dlogp is None else t64(dlogp)
        dl = torch.where(t >= 0, dl, 0.0)
        g = -dl[:, None] * self.p
        inside = (t >= 0) & (t < k)
        g[inside.nonzero()[:, 0], t[inside]] += dl[inside]
        if dentropy is not None:
            lp = torch.where(self.p > 0, self.lp, torch.where(self.p.isnan(), self.p, 0.0))
            g = g - t64(dentropy)[:, None] * self.p * (lp + self.h[:, None])
        g[self.none] = 0.0
        return g * self.s
