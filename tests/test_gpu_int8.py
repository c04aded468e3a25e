"""GPU parity of the 8-bit integer dense layers.  Every result is one bit pattern:
the quantised values are the exact quotients' roundings (checked in integers), the
sums are exact integers, and the rest is the declared float32 sequence."""

import math

import numpy as np
import pytest
import torch

import paper_1911_07384_amd as F
from gpu_util import note, require_gpu

pytestmark = pytest.mark.gpu


# ---- the oracle: integers, then the declared float32 sequence -----------------------

def quant_rows(x16: np.ndarray):
    """(q, scale) of a binary16 matrix by rows, with the quotient 127 x / max rounded
    in integers (binary16 values are multiples of 2^-24 below 2^40)."""
    finite = np.isfinite(x16).all(1)
    xi = np.where(np.isfinite(x16), x16.astype(np.float64), 0.0) * 2.0 ** 24
    xi = xi.astype(np.int64)
    top = np.abs(xi).max(1, keepdims=True)
    num, den = 127 * np.abs(xi), np.maximum(top, 1)
    k, r = num // den, num % den
    k += (2 * r > den) | ((2 * r == den) & (k % 2 == 1))
    q = np.where(finite[:, None], np.sign(xi) * k, 0).astype(np.int8)
    s = np.abs(x16).max(1).astype(np.float32) / np.float32(127.0)
    return q, np.where(finite, s, np.float32(np.nan)).astype(np.float32)


def product(qa, sa, qb, sb, bias=None):
    acc = (qa.astype(np.float64) @ qb.astype(np.float64).T)  # integers below 2^53
    with np.errstate(invalid="ignore", over="ignore"):
        y = (sa[:, None] * sb[None, :]).astype(np.float32) * acc.astype(np.float32)
        if bias is not None:
            y = y + bias.astype(np.float32)[None, :]
        return y.astype(np.float16)


def same(a, b):
    a, b = np.ascontiguousarray(a), np.ascontiguousarray(b)
    na, nb = np.isnan(a), np.isnan(b)
    return np.array_equal(na, nb) and np.array_equal(a[~na] + 0.0, b[~nb] + 0.0)


def acts(rows, cols, seed, scale=1.0):
    r = np.random.default_rng(seed)
    x = r.standard_normal((rows, cols)) * np.exp(0.5 * r.standard_normal((rows, 1))) * scale
    x *= np.where(r.random(cols) < 0.02, 8.0, 1.0)
    return x.astype(np.float16)


def gpu(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def run_quant(x, by):
    require_gpu()
    rows, cols = x.shape
    n, l = (rows, cols) if by == "rows" else (cols, rows)
    q, s = F.int8_operand(n, l)
    q.fill_(77)
    X = gpu(x)
    note(f"[gpu] int8 quant {by} {rows}x{cols}")
    if by == "rows":
        F.fp16_int8_quant_rows(rows, cols, X, q, s)
    else:
        F.fp16_int8_quant_cols(rows, cols, X, q, s,
                               F.workspace(F.fp16_int8_quant_workspace_bytes(rows, cols)))
    torch.cuda.synchronize()
    q, s = q.cpu().numpy(), s.cpu().numpy()
    assert (q[:, l:] == 0).all()  # the bytes past the row
    return q[:, :l], s


SIZES = [(1, 1), (1, 16), (3, 5), (7, 17), (16, 64), (5, 2048), (2, 2049), (3, 8192), (2, 8200),
         (1, 20011), (64, 63), (65, 64), (129, 200), (1111, 333), (4100, 24), (130, 1000)]


@pytest.mark.parametrize("by", ["rows", "cols"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: f"{s[0]}x{s[1]}")
def test_quantised_values(size, by):
    x = acts(*size, seed=sum(size))
    q, s = run_quant(x, by)
    qr, sr = quant_rows(x if by == "rows" else np.ascontiguousarray(x.T))
    assert np.array_equal(q, qr) and same(s, sr)


@pytest.mark.parametrize("by", ["rows", "cols"])
def test_halfway_and_special_values(by):
    """Every binary16 magnitude against several maxima (127 j, where quotients fall
    halfway, among them), zero rows, rows that are not finite, subnormal rows."""
    pats = np.arange(0, 0x7C00, 1, dtype=np.uint16).view(np.float16)
    rows = []
    for top in (127.0, 254.0, 1016.0, 635.0, 1.0, 65504.0, 2.0 ** -14 * 127 / 64, 0.3333):
        t = np.float16(top)
        v = pats[pats <= t].copy()
        v[::2] *= np.float16(-1)
        row = np.zeros(0x7C00 + 1, np.float16)
        row[:v.size] = v
        row[-1] = t
        rows.append(row)
    sub = np.zeros(0x7C00 + 1, np.float16)
    sub[:1024] = np.arange(1024, dtype=np.uint16).view(np.float16)
    zero, nan, inf, tiny = (np.zeros_like(sub) for _ in range(4))
    nan[7], inf[8], tiny[100] = np.nan, -np.inf, np.float16(2.0 ** -24)
    nan[9] = inf[9] = 3.0
    x = np.stack(rows + [sub, zero, nan, inf, tiny])
    q, s = run_quant(x if by == "rows" else np.ascontiguousarray(x.T), by)
    qr, sr = quant_rows(x)
    assert np.array_equal(q, qr) and same(s, sr)
    assert np.abs(qr).max() == 127 and np.isnan(sr[-3]) and np.isnan(sr[-2]) and sr[-4] == 0


# (m, n, k); test_product_choice.py holds the kernel each runs on
PRODUCTS = [(1, 1, 1), (1, 33, 100), (3, 1000, 2048), (16, 130, 4111), (2, 40, 131071),
            (17, 1, 15), (17, 40, 16), (64, 64, 128), (65, 129, 129), (128, 1000, 2048),
            (200, 77, 1337), (900, 700, 200), (2049, 2047, 300), (2100, 2056, 64),
            (1, 8192, 301), (16, 8193, 301), (1111, 2501, 1337), (2900, 3000, 700), (4001, 3601, 257), (3585, 3700, 128)]


@pytest.mark.parametrize("case", PRODUCTS, ids=lambda c: "x".join(map(str, c)))
def test_products(case):
    """Random bytes over the whole range, -128 among them; with a bias and without."""
    require_gpu()
    m, n, k = case
    r = np.random.default_rng(m + n + k)
    ld = F.fp16_int8_row_bytes(k)
    a, b = (np.zeros((rows, ld), np.int8) for rows in (m, n))
    a[:, :k] = r.integers(-128, 128, (m, k))
    b[:, :k] = r.integers(-128, 128, (n, k))
    # sums near the 32-bit limit in the first outputs
    a[0, :k] = -128
    b[0, :k] = -128
    sa, sb = (np.exp(r.standard_normal(rows)).astype(np.float32) * 1e-3 for rows in (m, n))
    sa[0] = sb[0] = 2.0 ** -16
    bias = r.standard_normal(n).astype(np.float16)
    A, B, SA, SB, BIAS = (gpu(t) for t in (a, b, sa, sb, bias))
    guard = 64
    for bi in (None, BIAS):
        buf = torch.full((m * n + guard,), 5.0, dtype=torch.float16, device="cuda")
        y = buf[:m * n].view(m, n)
        note(f"[gpu] int8 product {m}x{n}x{k} bias={bi is not None}")
        F.fp16_int8_matmul(m, n, k, A, SA, B, SB, bi, y)
        torch.cuda.synchronize()
        ref = product(a[:, :k], sa, b[:, :k], sb, None if bi is None else bias)
        assert same(y.cpu().numpy(), ref)
        assert (buf[m * n:] == 5).all()


DENSE = [(1, 64, 40), (1, 4096, 130), (3, 100, 1000), (13, 2048, 1000), (16, 9000, 33),
         # rows quantised by the product's workgroups up to 4 tokens, 16384 elements and
         # 8192 outputs, and just past that
         (4, 4096, 100), (4, 4097, 20), (2, 8192, 33), (3, 1000, 77), (5, 300, 20), (1, 65, 8192),
         (1, 65, 8193), (17, 72, 50), (100, 333, 77), (128, 2048, 1000), (515, 129, 300), (1111, 130, 257)]


def layer(t, i, o, seed=0):
    x, w, dy = acts(t, i, seed), acts(o, i, seed + 1, 0.05), acts(t, o, seed + 2, 1e-2)
    bias = (0.1 * np.random.default_rng(seed + 3).standard_normal(o)).astype(np.float16)
    return x, w, dy, bias


def run_layer(x, w, dy, bias, ws=None):
    require_gpu()
    (t, i), o = x.shape, w.shape[0]
    d = F.int8_dense_desc(t, i, o)
    ws = F.workspace(F.fp16_int8_dense_workspace_bytes(d)) if ws is None else ws
    X, W, DY = gpu(x), gpu(w), gpu(dy)
    B = None if bias is None else gpu(bias)
    wq, sw = F.int8_operand(o, i)
    wqt, swt = F.int8_operand(i, o)
    e = lambda *s: torch.full(s, float("nan"), dtype=torch.float16, device="cuda")
    y, dx, dw, db = e(t, o), e(t, i), e(o, i), e(o)
    note(f"[gpu] int8 layer {t}x{i}x{o}")
    F.fp16_int8_dense_weights(d, W, wq, sw, wqt, swt, ws)
    F.fp16_int8_dense_fwd(d, X, wq, sw, B, y, ws)
    F.fp16_int8_dense_bwd(d, X, DY, wqt, swt, dx, dw, db, ws)
    torch.cuda.synchronize()
    return [v.cpu().numpy() for v in (y, dx, dw, db)]


@pytest.mark.parametrize("size", DENSE, ids=lambda s: "x".join(map(str, s)))
def test_layer(size):
    x, w, dy, bias = layer(*size, seed=sum(size))
    T = np.ascontiguousarray
    y, dx, dw, db = run_layer(x, w, dy, bias)
    assert same(y, product(*quant_rows(x), *quant_rows(w), bias))
    assert same(dx, product(*quant_rows(dy), *quant_rows(T(w.T))))
    assert same(dw, product(*quant_rows(T(dy.T)), *quant_rows(T(x.T))))
    # the bias gradient: float32 partial sums of at most tokens terms, one rounding
    ref, mass = dy.astype(np.float64).sum(0), np.abs(dy.astype(np.float64)).sum(0)
    bound = np.abs(ref) * 2.0 ** -11 + 2.0 ** -25 + size[0] * 2.0 ** -24 * mass
    assert (np.abs(db.astype(np.float64) - ref) <= bound).all()


def test_parts_of_the_backward():
    """Each gradient alone is the one of the whole call."""
    x, w, dy, bias = layer(100, 96, 70)
    y, dx, dw, db = run_layer(x, w, dy, bias)
    d = F.int8_dense_desc(100, 96, 70)
    ws = F.workspace(F.fp16_int8_dense_workspace_bytes(d, F.INT8_BWD))
    wqt, swt = F.int8_operand(96, 70)
    wq, sw = F.int8_operand(70, 96)
    F.fp16_int8_dense_weights(d, gpu(w), wq, sw, wqt, swt,
                              F.workspace(F.fp16_int8_dense_workspace_bytes(d, F.INT8_WEIGHTS)))
    a, b = torch.empty(100, 96, dtype=torch.float16, device="cuda"), gpu(dw * 0)
    F.fp16_int8_dense_bwd(d, None, gpu(dy), wqt, swt, a, None, None, ws)
    F.fp16_int8_dense_bwd(d, gpu(x), gpu(dy), None, None, None, b, None, ws)
    torch.cuda.synchronize()
    assert same(a.cpu().numpy(), dx) and same(b.cpu().numpy(), dw)


def test_offsets_past_32_bits():
    """Quantisers of 2.2e9 elements and a product of as many outputs, compared in
    blocks on the device."""
    require_gpu()
    rows, cols = 70001, 31003
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty((rows, cols), dtype=torch.float16, device="cuda").normal_(generator=g)
    assert x.numel() > 2 ** 31
    for by in ("rows", "cols"):
        n, l = (rows, cols) if by == "rows" else (cols, rows)
        q, s = F.int8_operand(n, l)
        note(f"[gpu] int8 quant {by} {rows}x{cols}")
        if by == "rows":
            F.fp16_int8_quant_rows(rows, cols, x, q, s)
        else:
            F.fp16_int8_quant_cols(rows, cols, x, q, s,
                                   F.workspace(F.fp16_int8_quant_workspace_bytes(rows, cols)))
        torch.cuda.synchronize()
        for a in list(range(0, n - 4096, 8192)) + [n - 4096]:
            b = min(n, a + 4096)
            t = x[a:b] if by == "rows" else x[:, a:b].t().contiguous()
            top = t.abs().amax(1, keepdim=True).double()
            # (quotients in float64 are within 2^-52 of halfway ones or exactly there)
            assert torch.equal(q[a:b, :l], (127.0 * t.double() / top).round().to(torch.int8))
            assert not q[a:b, l:].any()
            assert torch.equal(s[a:b].cpu(), top[:, 0].float().cpu() / np.float32(127.0))
        del q, s
    del x, t
    m, n, k = 70001, 31003, 33
    (qa, sa), (qb, sb) = F.int8_operand(m, k), F.int8_operand(n, k)
    for q, s in ((qa, sa), (qb, sb)):
        q.zero_()
        q[:, :k] = torch.randint(-127, 128, (len(q), k), generator=g, device="cuda").to(torch.int8)
        s.uniform_(0.001, 0.002, generator=g)
    y = torch.empty((m, n), dtype=torch.float16, device="cuda")
    note(f"[gpu] int8 product {m}x{n}x{k} {F.fp16_int8_kernel(m, n, k)}")
    F.fp16_int8_matmul(m, n, k, qa, sa, qb, sb, None, y)
    torch.cuda.synchronize()
    bt = qb.float().t().contiguous()
    for a in list(range(0, m - 4096, 8192)) + [m - 4096]:
        b = min(m, a + 4096)
        acc = qa[a:b].float() @ bt  # integers below 2^24
        assert torch.equal(y[a:b], (sa[a:b, None] * sb[None, :] * acc).half())


def test_rows_that_are_not_finite_stay_apart():
    """A token with a NaN makes its own outputs NaN, and no other token's."""
    x, w, dy, bias = layer(40, 64, 32)
    clean = run_layer(x, w, dy, bias)
    x2 = x.copy()
    x2[7, 3], x2[9, 0] = np.nan, np.inf
    y = run_layer(x2, w, dy, bias)[0]
    assert np.isnan(y[[7, 9]]).all()
    keep = [i for i in range(40) if i not in (7, 9)]
    assert same(y[keep], clean[0][keep])


def test_gradients_on_the_grid_against_differences():
    """Values that the 8-bit grid holds exactly: the layer is then linear, so a
    difference of the float64 loss <dy, y> along one weight or input is its gradient."""
    r = np.random.default_rng(0)
    t, i, o = 24, 32, 20
    x, w, dy = (r.integers(-100, 101, s).astype(np.float16) for s in ((t, i), (o, i), (t, o)))
    for m in (x, w, dy):  # every row and every column has the maximum 127
        n = max(m.shape)
        m[np.arange(n) % m.shape[0], np.arange(n) % m.shape[1]] = 127
    scale = np.float16(2.0 ** -10)
    x, w, dy = x * scale, w * scale, dy * scale
    y, dx, dw, _ = run_layer(x, w, dy, None)
    loss = lambda a, b: float((dy.astype(np.float64) * (a.astype(np.float64) @ b.astype(np.float64).T)).sum())
    half = lambda v: abs(v) * 2.0 ** -11 + 2.0 ** -25  # one rounding of the result
    f32 = 3 * 2.0 ** -24                               # scale, sum and product in float32
    for _ in range(20):
        j, k, n = r.integers(0, o), r.integers(0, i), r.integers(0, t)
        h = 2.0 ** -6
        for base, got, at in ((w, dw, (j, k)), (x, dx, (n, k))):
            up, dn = base.astype(np.float64), base.astype(np.float64)
            up[at] += h
            dn[at] -= h
            d = (loss(x, up) - loss(x, dn) if base is w else loss(up, w) - loss(dn, w)) / (2 * h)
            assert abs(float(got[at]) - d) <= half(d) + f32 * abs(d) + 1e-12


def test_same_bits_in_a_graph_and_on_another_stream():
    require_gpu()
    x, w, dy, bias = layer(77, 130, 90, 5)
    ref = run_layer(x, w, dy, bias)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        assert all(same(a, b) for a, b in zip(run_layer(x, w, dy, bias), ref))
    d = F.int8_dense_desc(77, 130, 90)
    ws = F.workspace(F.fp16_int8_dense_workspace_bytes(d))
    X, W, DY, B = (gpu(v) for v in (x, w, dy, bias))
    wq, sw = F.int8_operand(90, 130)
    wqt, swt = F.int8_operand(130, 90)
    out = [torch.empty(v.shape, dtype=torch.float16, device="cuda") for v in ref]

    def go():
        F.fp16_int8_dense_weights(d, W, wq, sw, wqt, swt, ws)
        F.fp16_int8_dense_fwd(d, X, wq, sw, B, out[0], ws)
        F.fp16_int8_dense_bwd(d, X, DY, wqt, swt, out[1], out[2], out[3], ws)

    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        go()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        go()
    for k in range(3):
        x, w, dy, bias = layer(77, 130, 90, 50 + k)
        for t, v in ((X, x), (W, w), (DY, dy), (B, bias)):
            t.copy_(torch.from_numpy(v))
        for t in out:
            t.fill_(9.0)
        g.replay()
        torch.cuda.synchronize()
        got = [t.cpu().numpy() for t in out]
        assert all(same(a, b) for a, b in zip(got, run_layer(x, w, dy, bias))), k
