"""Host-side checks of the dense head's entry points: every call here carries an invalid
argument (or asks for nothing), so nothing is launched and the fake addresses are not
followed."""

import ctypes

import pytest
import torch

import paper_1911_07384_amd as F

OK, NULL, SHAPE, LAYOUT, MISALIGNED, ALIASING, WORKSPACE = 0, 1, 2, 3, 4, 5, 6
A, B, C, D, E, G, H, R, W = (0x1000000000 * k for k in range(1, 10))  # far apart, aligned
BIG = 1 << 40
NAN, INF = float("nan"), float("inf")


def dropout(n=1000, x=A, res=None, y=B, p=0.5, rng=R):
    return F.lib().fp16_dropout(n, x, res, y, p, rng, 0, None)


def test_dropout_refusals():
    assert dropout(n=0, x=None, y=None, rng=None) == OK
    for p in (-0.1, 1.1, NAN, INF):
        assert dropout(p=p) == SHAPE and dropout(n=0, p=p) == SHAPE
    assert dropout(n=1 << 34) == SHAPE
    assert dropout(x=None) == NULL and dropout(y=None) == NULL and dropout(rng=None) == NULL
    assert dropout(x=A + 2) == MISALIGNED and dropout(y=B + 8) == MISALIGNED
    assert dropout(res=C + 4) == MISALIGNED and dropout(rng=R + 4) == MISALIGNED
    assert dropout(y=A + 16) == ALIASING and dropout(y=A + 1984) == ALIASING
    assert dropout(res=C, y=C + 16) == ALIASING and dropout(rng=B + 8) == ALIASING
    # in place on x, but over the residual besides
    assert dropout(y=A, res=A + 16) == ALIASING
    assert F.lib().fp16_rng_advance(None, 1, None) == NULL
    assert F.lib().fp16_rng_advance(R + 4, 1, None) == MISALIGNED


def desc(tokens=24, inputs=40, outputs=56, act="none", drop=0.0):
    return F.dense_desc(tokens, inputs, outputs, act, drop)


def fwd(d=None, x=A, w=B, bias=None, res=None, rng=None, y=C, z=None, ws=W, n=BIG, ref=True):
    d = desc() if d is None else d
    return F.lib().fp16_dense_fwd(ctypes.byref(d) if ref else None, x, w, bias, res, rng, y, z, ws,
                                  n, None)


def bwd(d=None, x=A, w=B, z=None, dy=C, rng=None, dx=D, dw=E, db=None, ws=W, n=BIG, ref=True):
    d = desc() if d is None else d
    return F.lib().fp16_dense_bwd(ctypes.byref(d) if ref else None, x, w, z, dy, rng, dx, dw, db,
                                  ws, n, None)


BAD = [desc(tokens=0), desc(inputs=0), desc(outputs=0), desc(tokens=-1), desc(tokens=(1 << 20) + 1),
       desc(inputs=(1 << 20) + 1), desc(outputs=(1 << 20) + 1), desc(act=4), desc(act=-1),
       desc(drop=-0.1), desc(drop=1.5), desc(drop=NAN), desc(tokens=1 << 20, inputs=1 << 14),
       desc(tokens=1 << 20, outputs=1 << 14), desc(inputs=1 << 20, outputs=1 << 14)]


def test_dense_forward_refusals():
    assert fwd(ref=False) == NULL
    for d in BAD:
        assert fwd(d) == SHAPE and bwd(d, z=G) == SHAPE
        assert F.lib().fp16_dense_workspace_bytes(ctypes.byref(d), 0) == 0
        assert F.lib().fp16_dense_workspace_bytes(ctypes.byref(d), 1) == 0
    assert fwd(x=None) == NULL and fwd(w=None) == NULL and fwd(y=None) == NULL
    assert fwd(desc(drop=0.5)) == NULL  # no generator
    for k in ("x", "w", "bias", "res", "y", "z"):
        assert fwd(**{k: G + 8}) == MISALIGNED, k
    assert fwd(rng=R + 4) == MISALIGNED
    assert fwd(y=A) == ALIASING and fwd(y=B) == ALIASING and fwd(z=C) == ALIASING
    assert fwd(bias=C + 16) == ALIASING and fwd(res=C + 16) == ALIASING
    assert fwd(z=G, res=G) == ALIASING and fwd(z=A) == ALIASING
    assert fwd(desc(drop=0.5), rng=C + 8) == ALIASING
    # a residual updated in place is taken, and refused only for the overlap behind it
    assert fwd(res=C, z=C) == ALIASING


def test_dense_backward_refusals():
    assert bwd(ref=False) == NULL and bwd(dy=None) == NULL
    assert bwd(x=None) == NULL and bwd(w=None) == NULL
    assert bwd(desc(act="relu")) == NULL and bwd(desc(drop=0.5)) == NULL
    assert bwd(dx=None, dw=None) == OK  # nothing is asked for
    for k in ("x", "w", "dy", "dx", "dw", "db"):
        assert bwd(**{k: G + 8}) == MISALIGNED, k
    assert bwd(desc(act="gelu"), z=G + 8) == MISALIGNED
    gelu = desc(act="gelu")
    need = F.fp16_dense_workspace_bytes(gelu, F.DENSE_BWD)
    assert need >= 24 * 56 * 2
    assert bwd(gelu, z=G, n=need - 1) == WORKSPACE and bwd(gelu, z=G, ws=None) == WORKSPACE
    assert bwd(gelu, z=G, ws=W + 8) == MISALIGNED
    assert bwd(dx=A) == ALIASING and bwd(dw=B) == ALIASING and bwd(dx=C) == ALIASING
    assert bwd(dw=D + 16) == ALIASING and bwd(db=D) == ALIASING and bwd(db=E + 32) == ALIASING
    assert bwd(gelu, z=D) == ALIASING and bwd(gelu, z=W) == ALIASING
    assert bwd(gelu, z=G, dx=W) == ALIASING
    assert bwd(desc(drop=0.5), rng=D + 8) == ALIASING
    assert F.lib().fp16_dense_workspace_bytes(None, 0) == 0
    d = desc()
    assert F.lib().fp16_dense_workspace_bytes(ctypes.byref(d), 2) == 0
    assert F.lib().fp16_dense_workspace_bytes(ctypes.byref(d), -1) == 0


def logp(d=None, z=A, tok=B, lp=C, st=D, ti=None, tl=None, ws=W, n=BIG, ref=True):
    d = F.logprob_desc(10, 100) if d is None else d
    return F.lib().fp16_logprobs(ctypes.byref(d) if ref else None, z, tok, lp, st, ti, tl, ws, n,
                                 None)


def logb(d=None, z=A, tok=B, st=C, dl=D, dh=E, dz=G, ref=True):
    d = F.logprob_desc(10, 100) if d is None else d
    return F.lib().fp16_logprobs_bwd(ctypes.byref(d) if ref else None, z, tok, st, dl, dh, dz, None)


def test_logprob_refusals():
    L = F.logprob_desc
    for d in [L(0, 10), L(10, 0), L(-1, 5), L(1 << 24, 1), L(1, (1 << 20) + 1), L(4, 10, stride=9),
              L(4, 10, stride=(1 << 21) + 1), L((1 << 24) - 1, 4096), L(4, 10, scale=0.0),
              L(4, 10, scale=-1.0), L(4, 10, scale=NAN), L(4, 10, scale=INF), L(4, 10, scale=2e30), L(4, 10, top=-1),
              L(4, 10, top=11), L(4, 100, top=65)]:
        assert logp(d, ti=E, tl=G) == SHAPE and logb(d) == SHAPE
        assert F.lib().fp16_logprobs_workspace_bytes(ctypes.byref(d)) == 0
    assert F.lib().fp16_logprobs_workspace_bytes(None) == 0
    assert logp(ref=False) == NULL and logp(z=None) == NULL and logp(st=None) == NULL
    assert logp(tok=None) == NULL  # a log probability of which class?
    top = L(10, 100, top=5)
    assert logp(top, ti=E) == NULL and logp(top, tl=E) == NULL
    for k in ("z", "tok", "lp", "st"):
        assert logp(**{k: H + 8}) == MISALIGNED, k
    assert logp(top, ti=E + 4, tl=G) == MISALIGNED and logp(top, ti=E, tl=G + 4) == MISALIGNED
    assert logp(lp=A) == ALIASING and logp(st=B) == ALIASING and logp(st=C + 32) == ALIASING
    assert logp(top, ti=E, tl=E + 16) == ALIASING and logp(top, ti=A + 1984, tl=E) == ALIASING
    long = L(1, 1 << 20, top=64)
    need = F.fp16_logprobs_workspace_bytes(long)
    assert need > 0
    assert logp(long, ti=E, tl=G, n=need - 1) == WORKSPACE
    assert logp(long, ti=E, tl=G, ws=None) == WORKSPACE
    assert logp(long, ti=E, tl=G, ws=W + 8) == MISALIGNED
    assert logp(long, ti=E, tl=W, ) == ALIASING


def test_logprob_backward_refusals():
    assert logb(ref=False) == NULL
    assert logb(z=None) == NULL and logb(st=None) == NULL and logb(dz=None) == NULL
    assert logb(dl=None, dh=None) == NULL and logb(tok=None) == NULL
    for k in ("z", "tok", "st", "dl", "dh", "dz"):
        assert logb(**{k: H + 4}) == MISALIGNED, k
    assert logb(dz=A + 16) == ALIASING and logb(dz=B) == ALIASING and logb(dz=C) == ALIASING
    assert logb(dz=D) == ALIASING and logb(dz=E) == ALIASING


def test_binding_checks(monkeypatch):
    monkeypatch.setattr(F, "_device", lambda: -1)  # (a CPU tensor's)
    cpu = lambda *s, t=torch.float16: torch.zeros(s, dtype=t)
    d = F.dense_desc(4, 8, 16)
    with pytest.raises(ValueError, match="w has"):
        F.fp16_dense_fwd(d, cpu(4, 8), cpu(8, 8), None, None, cpu(4, 16), stream=0)
    with pytest.raises(TypeError):
        F.fp16_dense_fwd(d, cpu(4, 8), cpu(16, 8, t=torch.float32), None, None, cpu(4, 16), stream=0)
    with pytest.raises(ValueError, match="contiguous"):
        F.fp16_dense_fwd(d, cpu(8, 4).t(), cpu(16, 8), None, None, cpu(4, 16), stream=0)
    with pytest.raises(ValueError, match="dx has"):
        F.fp16_dense_bwd(d, cpu(4, 8), cpu(16, 8), None, cpu(4, 16), cpu(3, 8), None, stream=0)
    with pytest.raises(KeyError):
        F.dense_desc(4, 8, 16, act="tanh")
    with pytest.raises(ValueError, match="rng has"):
        F.fp16_dropout(cpu(8), None, cpu(8), 0.5, cpu(1, t=torch.int64), stream=0)
    with pytest.raises(TypeError):
        F.fp16_dropout(cpu(8), None, cpu(8), 0.5, cpu(2, t=torch.int32), stream=0)
    with pytest.raises(ValueError, match="tokens has"):
        F.fp16_logprobs(F.logprob_desc(4, 8), cpu(4, 8), cpu(3, t=torch.int32),
                        cpu(4, t=torch.float32), cpu(12, t=torch.float32), stream=0)
    with pytest.raises(ValueError, match="z has"):
        F.fp16_logprobs(F.logprob_desc(4, 8, stride=9), cpu(4, 8), None, None,
                        cpu(12, t=torch.float32), stream=0)
    with pytest.raises(TypeError):
        F.fp16_logprobs_bwd(F.logprob_desc(4, 8), cpu(4, 8), None, cpu(12, t=torch.float32), None,
                            cpu(4), cpu(4, 8), stream=0)
    s = F.rng_state((1 << 64) - 1, 1 << 63, device="cpu")
    assert s.tolist() == [-1, -(1 << 63)]


def test_tensors_of_another_device(monkeypatch):
    """Arguments that are right but for their device are refused before the call."""
    monkeypatch.setattr(F, "_device", lambda: 0)
    h = lambda *s: torch.zeros(s, dtype=torch.float16)
    f = lambda *s: torch.zeros(s, dtype=torch.float32)
    rng = F.rng_state(1, device="cpu")
    d, lp = F.dense_desc(4, 8, 16), F.logprob_desc(4, 8)
    for call in (lambda: F.fp16_rng_advance(rng, stream=0),
                 lambda: F.fp16_dropout(A, None, B, 0.5, rng, n=8, stream=0),
                 lambda: F.fp16_dropout(h(8), None, B, 0.5, R, stream=0),
                 lambda: F.fp16_dense_fwd(d, A, B, None, h(4, 16), C, stream=0),
                 lambda: F.fp16_dense_fwd(d, A, B, None, None, C, ws=f(8), stream=0),
                 lambda: F.fp16_dense_bwd(d, A, B, None, C, D, h(16, 8), stream=0),
                 lambda: F.fp16_logprobs(lp, A, None, None, f(12), stream=0),
                 lambda: F.fp16_logprobs_bwd(lp, A, None, B, f(4), None, C, stream=0)):
        with pytest.raises(ValueError, match="current device"):
            call()
