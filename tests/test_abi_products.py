"""Host-side checks of the entry points for orthogonalised momentum and 8-bit dense
layers: every call here carries an invalid argument, so nothing is launched (the
pointers are fake addresses that validation must not follow)."""

import ctypes

import numpy as np
import pytest

import paper_1911_07384_amd as F
import test_gpu_int8 as oracle8

OK, NULL, SHAPE, LAYOUT, MISALIGNED, ALIASING, WORKSPACE = 0, 1, 2, 3, 4, 5, 6
A, B, C, D, E, W = (0x10000000 * k for k in range(1, 7))  # far apart, 16-byte aligned
BIG = 1 << 34


def _list(*p):
    return (ctypes.c_void_p * max(len(p), 1))(*p)


def orth(shapes=((64, 64),), x=(A,), y=(B,), steps=5, coef=None, products=1, ws=W, wsb=BIG,
         count=None):
    d = F.muon_descs(shapes)
    c = None if coef is None else (ctypes.c_float * len(coef))(*coef)
    return F.lib().fp16_orthogonalize(len(shapes) if count is None else count, d, _list(*x),
                                      _list(*y), steps, c, products, ws, wsb, None)


def test_orthogonalize_refusals():
    assert orth(count=0) == OK  # a no-op: nothing is read
    assert F.lib().fp16_orthogonalize(0, None, None, None, 5, None, 1, None, 0, None) == OK
    assert orth(count=-1) == SHAPE and orth(count=1025) == SHAPE
    assert F.lib().fp16_orthogonalize(1, None, _list(A), _list(B), 5, None, 1, W, BIG, None) == NULL
    assert F.lib().fp16_orthogonalize(1, F.muon_descs([(8, 8)]), None, _list(B), 5, None, 1, W, BIG,
                                      None) == NULL
    assert orth(x=(None,)) == NULL and orth(y=(None,)) == NULL
    for s in [(0, 64), (64, 0), (-1, 64), (65537, 1), (1, 65537), (16385, 16385), (65536, 16384),
              (64, 64, float("nan")), (64, 64, float("inf"))]:
        assert orth(shapes=(s,)) == SHAPE, s
    for kw in [dict(steps=0), dict(steps=33), dict(steps=-1), dict(products=0), dict(products=2),
               dict(coef=[1.0, float("nan"), 0.0] * 5)]:
        assert orth(**kw) == SHAPE, kw
    # an element's alignment is enough for matrices, the workspace needs 16 bytes
    assert orth(x=(A + 1,)) == MISALIGNED and orth(y=(B + 1,)) == MISALIGNED
    assert orth(ws=W + 8) == MISALIGNED
    need = F.fp16_muon_workspace_bytes(F.muon_descs([(64, 64)]), 1)
    assert need > 0
    assert orth(wsb=need - 1) == WORKSPACE and orth(ws=None) == WORKSPACE


def test_orthogonalize_aliasing():
    two = ((64, 64), (64, 64))
    n = 64 * 64 * 2
    assert orth(y=(A + 2,)) == ALIASING and orth(y=(A + n - 2,)) == ALIASING
    assert orth(two, (A, B), (C, C)) == ALIASING          # the same result twice
    assert orth(two, (A, B), (C, C + n - 2)) == ALIASING
    assert orth(two, (A, B), (B, C)) == ALIASING          # another's input
    assert orth(y=(W + 64,)) == ALIASING and orth(x=(W + 64,)) == ALIASING


def test_muon_refusals():
    d = F.muon_descs([(64, 64)])

    def call(w=A, g=B, m=C, lr=0.1, mu=0.9, wd=0.0, ws=W, wsb=BIG, steps=5, products=1):
        return F.lib().fp16_muon_step(1, d, _list(w), _list(g), _list(m), lr, mu, wd, 1, steps, None,
                                      products, ws, wsb, None)

    assert call(w=None) == NULL and call(g=None) == NULL and call(m=None) == NULL
    assert F.lib().fp16_muon_step(1, d, _list(A), _list(B), None, 0.1, 0.9, 0.0, 1, 5, None, 1, W,
                                  BIG, None) == NULL
    nan = float("nan")
    assert call(lr=nan) == SHAPE and call(mu=nan) == SHAPE and call(wd=float("inf")) == SHAPE
    assert call(steps=0) == SHAPE and call(products=4) == SHAPE
    assert call(m=C + 1) == MISALIGNED and call(ws=W + 2) == MISALIGNED
    assert call(wsb=100) == WORKSPACE
    assert call(g=A) == ALIASING and call(m=A) == ALIASING and call(m=B) == ALIASING
    assert call(m=A + 100) == ALIASING and call(w=W) == ALIASING


def test_workspace_queries():
    f = F.fp16_muon_workspace_bytes
    one, three = (f(F.muon_descs([(512, 512)]), p) for p in (1, 3))
    assert 0 < one < three
    assert f(F.muon_descs([(512, 512)]), 2) == 0 and f(F.muon_descs([(0, 512)]), 1) == 0
    assert F.fp16_muon_kernels(F.muon_descs([(0, 512)])) == ""
    assert F.fp16_int8_quant_workspace_bytes(0, 4) == 0 and F.fp16_int8_quant_workspace_bytes(9, 4) > 0
    assert F.fp16_int8_row_bytes(0) == 0
    assert [F.fp16_int8_row_bytes(n) for n in (1, 16, 17, 131071)] == [16, 16, 32, 131072]
    d = F.int8_dense_desc(100, 64, 32)
    assert all(F.fp16_int8_dense_workspace_bytes(d, c) > 0 for c in range(3))
    assert F.lib().fp16_int8_dense_workspace_bytes(ctypes.byref(d), 3) == 0
    assert F.lib().fp16_int8_dense_workspace_bytes(None, 0) == 0
    assert F.fp16_int8_dense_workspace_bytes(F.int8_dense_desc(0, 64, 32)) == 0
    # a single token needs none
    assert F.fp16_int8_dense_workspace_bytes(F.int8_dense_desc(1, 4096, 64), F.INT8_FWD) == 0


def test_quantiser_refusals():
    rows = lambda r=8, c=8, x=A, q=B, s=C: F.lib().fp16_int8_quant_rows(r, c, x, q, s, None)
    cols = lambda r=8, c=8, x=A, q=B, s=C, ws=W, n=BIG: F.lib().fp16_int8_quant_cols(
        r, c, x, q, s, ws, n, None)
    for f in (rows, cols):
        assert f(r=0) == SHAPE and f(c=0) == SHAPE and f(r=1 << 22) == SHAPE and f(c=-1) == SHAPE
        assert f(r=(1 << 22) - 1, c=(1 << 22) - 1) == SHAPE
        assert f(x=None) == NULL and f(q=None) == NULL and f(s=None) == NULL
        assert f(x=A + 2) == MISALIGNED and f(q=B + 8) == MISALIGNED and f(s=C + 4) == MISALIGNED
        assert f(q=A) == ALIASING and f(s=A + 16) == ALIASING and f(s=B + 16) == ALIASING
    assert cols(ws=None) == WORKSPACE and cols(n=1) == WORKSPACE and cols(ws=W + 4) == MISALIGNED
    assert cols(ws=A) == ALIASING


def test_matmul_refusals():
    def mm(m=20, n=24, k=40, a=A, sa=B, b=C, sb=D, bias=None, y=E):
        return F.lib().fp16_int8_matmul(m, n, k, a, sa, b, sb, bias, y, None)

    for kw in [dict(m=0), dict(n=0), dict(k=0), dict(k=131072), dict(m=1 << 22), dict(n=1 << 22),
               dict(m=(1 << 21), n=(1 << 21))]:
        assert mm(**kw) == SHAPE, kw
        assert F.fp16_int8_kernel(kw.get("m", 20), kw.get("n", 24), kw.get("k", 40)) == ""
    for name in ("a", "sa", "b", "sb", "y"):
        assert mm(**{name: None}) == NULL, name
        assert mm(**{name: A + 8}) == MISALIGNED, name
    assert mm(bias=W + 2) == MISALIGNED
    for other in (A, B, C, D):
        assert mm(y=other) == ALIASING
    assert mm(bias=E + 16) == ALIASING


def test_dense_refusals():
    d = F.int8_dense_desc(100, 64, 32)
    lib, ref = F.lib(), ctypes.byref(d)
    fwd = lambda x=A, wq=B, sw=C, bias=None, y=D, ws=W, n=BIG, p=ref: lib.fp16_int8_dense_fwd(
        p, x, wq, sw, bias, y, ws, n, None)
    assert fwd(p=None) == NULL and fwd(x=None) == NULL and fwd(y=None) == NULL
    assert fwd(ws=None) == WORKSPACE and fwd(n=8) == WORKSPACE and fwd(ws=W + 8) == MISALIGNED
    assert fwd(y=A) == ALIASING and fwd(y=W) == ALIASING and fwd(x=W) == ALIASING
    assert fwd(bias=A + 2) == MISALIGNED
    for bad in [(0, 64, 32), (100, 131072, 32), (100, 64, 0), (131072, 64, 32)]:
        assert fwd(p=ctypes.byref(F.int8_dense_desc(*bad))) == SHAPE
    wts = lambda w=A, wq=B, sw=C, wqt=D, swt=E, ws=W, n=BIG: lib.fp16_int8_dense_weights(
        ref, w, wq, sw, wqt, swt, ws, n, None)
    assert wts(w=None) == NULL and wts(wqt=None) == NULL and wts(swt=None) == NULL
    assert wts(ws=None) == WORKSPACE and wts(wq=A) == ALIASING and wts(wqt=B) == ALIASING
    assert wts(wqt=D + 4) == MISALIGNED
    X = 0x70000000
    bwd = lambda x=A, dy=B, wqt=C, swt=D, dx=E, dw=X, db=None, ws=W, n=BIG: lib.fp16_int8_dense_bwd(
        ref, x, dy, wqt, swt, dx, dw, db, ws, n, None)
    assert bwd(dy=None) == NULL and bwd(x=None) == NULL and bwd(wqt=None) == NULL
    assert bwd(swt=None) == NULL and bwd(dw=None, db=X) == NULL
    assert bwd(n=64) == WORKSPACE and bwd(dx=B) == ALIASING and bwd(dw=A) == ALIASING
    assert bwd(dw=E + 32) == ALIASING and bwd(db=E) == ALIASING and bwd(dw=X + 2) == MISALIGNED


def test_binding_checks():
    with pytest.raises(ValueError):
        F.fp16_orthogonalize(F.muon_descs([(8, 8)]), [A], [B, C], ws=W, ws_bytes=0, stream=0)
    with pytest.raises(ValueError):  # (a workspace for two, tensors for one)
        F.fp16_orthogonalize(F.muon_descs([(8, 8)] * 2), [A], [B], ws=W, ws_bytes=0, stream=0)
    F.fp16_orthogonalize(F.muon_descs([]), [], [], stream=0)  # nothing to do
    F.fp16_muon_step(F.muon_descs([]), [], [], [], stream=0)
    with pytest.raises(ValueError):
        F.fp16_orthogonalize(F.muon_descs([(8, 8)]), [A], [B], coef=(1.0, 2.0), ws=W, ws_bytes=0,
                             stream=0)
    with pytest.raises(F.Fp16Error, match="FP16_ERR_WORKSPACE"):
        F.fp16_orthogonalize(F.muon_descs([(8, 8)]), [A], [B], ws=W, ws_bytes=0, stream=0)


def test_the_quantisers_oracle():
    """quant_rows of the GPU tests against exact rationals."""
    from fractions import Fraction
    r = np.random.default_rng(0)
    x = (r.standard_normal((6, 40)) * 2.0 ** r.integers(-20, 10, (6, 1))).astype(np.float16)
    x[0, :3] = [127.0, 0.5, -1.5]  # halves of 127 / 127
    x[0, 3:] = np.clip(x[0, 3:], -100, 100)
    x[1] = 0
    q, s = oracle8.quant_rows(x)
    for i in range(6):
        top = max(Fraction(float(v)) for v in np.abs(x[i]))
        for j in range(40):
            want = round(127 * Fraction(float(x[i, j])) / top) if top else 0
            assert q[i, j] == want
        assert s[i] == np.float32(np.float32(float(top)) / np.float32(127))


def test_a_workspace_by_default_serves_either_call_by_default():
    """Queried without a number of products it holds one or three: each call, with its
    own default, gets past the workspace to the next refusal (an overlap)."""
    for shapes in ([(64, 64)], [(512, 4608)] * 3, [(1024, 4096)], [(70, 80), (700, 300)]):
        d = F.muon_descs(shapes)
        need = F.fp16_muon_workspace_bytes(d)
        assert need == max(F.fp16_muon_workspace_bytes(d, 1), F.fp16_muon_workspace_bytes(d, 3))
        far = lambda base: [base + (1 << 28) * i for i in range(len(shapes))]
        with pytest.raises(F.Fp16Error, match="FP16_ERR_ALIASING"):
            F.fp16_orthogonalize(d, far(1 << 40), far(2 << 40), ws=1 << 40, ws_bytes=need, stream=0)
        with pytest.raises(F.Fp16Error, match="FP16_ERR_ALIASING"):
            F.fp16_muon_step(d, far(1 << 40), far(2 << 40), far(3 << 40), ws=1 << 40, ws_bytes=need,
                             stream=0)
