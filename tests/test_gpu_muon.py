"""GPU parity of fp16_orthogonalize and fp16_muon_step against float64.

Bars (2-norm, relative).  A step is X <- p(X) on the singular values with
p(s) = as + bs^3 + cs^5, |p'| <= 3.9 up to s = 1.2, so an error entering at step k
is multiplied by at most 3.9^(steps - k).
  products = 3: operands carry 22 bits, an error of a few 2^-22 a step; five steps
    give 2^-22 * 3 * (3.9^5 - 1) / 2.9 = 2.2e-4 at most; plus the rounding of the
    result, 2^-11.
  products = 1: A, B and X as operands are each rounded by up to 2^-11 in the last
    step, and that is multiplied by at most 3.9: 3 * 3.9 * 2^-11 = 5.8e-3 (what
    earlier steps leave is within that: X itself keeps 22 bits); plus 2^-11.
"""

import math

import numpy as np
import pytest
import torch

import oracle
import paper_1911_07384_amd as F
from gpu_util import dev, host, note, require_gpu

pytestmark = pytest.mark.gpu

QUINTIC = (3.4445, -4.7750, 2.0315)
BAR = {1: 3 * 3.9 * 2.0 ** -11 + 2.0 ** -11,
       3: 2.0 ** -22 * 3 * (3.9 ** 5 - 1) / 2.9 + 2.0 ** -11}


def matrix(rows, cols, seed, kind="noisy", scale=1e-3):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((rows, cols), generator=g, dtype=torch.float64)
    if kind == "noisy":  # a few strong directions over noise, as gradients are
        r = max(1, min(rows, cols) // 16)
        u = torch.randn((rows, r), generator=g, dtype=torch.float64)
        v = torch.randn((r, cols), generator=g, dtype=torch.float64)
        x = 0.1 * x + (u * torch.logspace(0, -1, r, dtype=torch.float64)) @ v / math.sqrt(r)
    return (x * scale).half()


def ns64(u, steps=5, coef=None, scale=1.0):
    """Newton-Schulz in float64 on the device (or 0 for a zero matrix)."""
    x = u.double().cuda()
    n = x.norm()
    if n == 0:
        return x
    x = x / n
    if x.shape[0] > x.shape[1]:
        x = x.t().contiguous()
    for s in range(steps):
        a, b, c = QUINTIC if coef is None else coef[s] if isinstance(coef, list) else coef
        p = x @ x.t()
        x = a * x + (b * p + c * (p @ p)) @ x
    return (x if u.shape[0] <= u.shape[1] else x.t()) * scale


def off(got, ref):
    n = ref.norm().item()
    return (got.double() - ref).norm().item() / n if n else got.double().norm().item()


def orth(xs, products, steps=5, coef=None, scales=None, ws=None, out=None):
    require_gpu()
    scales = scales or [1.0] * len(xs)
    d = F.muon_descs([(x.shape[0], x.shape[1], s) for x, s in zip(xs, scales)])
    X = [x.cuda() for x in xs]
    Y = out or [torch.full_like(x, float("nan")) for x in X]
    ws = F.workspace(F.fp16_muon_workspace_bytes(d, products)) if ws is None else ws
    note(f"[gpu] orthogonalize {[tuple(x.shape) for x in xs][:6]} products={products}")
    F.fp16_orthogonalize(d, X, Y, steps, coef, products, ws)
    torch.cuda.synchronize()
    return Y


SHAPES = [(1, 1), (1, 7), (5, 1), (2, 2), (3, 3), (8, 8), (16, 200), (200, 16), (63, 65), (64, 64),
          (65, 63), (64, 147), (147, 64), (64, 576), (129, 300), (256, 256), (300, 520), (1000, 257),
          (257, 1000), (512, 512),
          # one workgroup each: up to 64 by 1024, tiles of 32 by the longer side
          (64, 31), (33, 32), (32, 33), (64, 65), (1, 1024), (1023, 1), (64, 1024), (1024, 64),
          (576, 64), (40, 999), (999, 40), (64, 1025)]


@pytest.mark.parametrize("products", [1, 3])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"{s[0]}x{s[1]}")
def test_shapes(shape, products):
    x = matrix(*shape, seed=sum(shape))
    y, = orth([x], products)
    assert off(y, ns64(x)) <= BAR[products]


# sets that between them run A, B and X' on every tile that each is offered
# (test_product_choice.py holds that)
SETS = [[(96, 700)], [(1034, 16)], [(16, 1475)], [(1989, 16)], [(76, 65)], [(16, 3534)] * 4,
        [(725, 709)] * 8, [(751, 651)] * 8, [(782, 818)] * 8, [(911, 994)] * 8, [(654, 935)] * 8,
        [(1223, 450)] * 8, [(1248, 1043)] * 8, [(1322, 1324)] * 8, [(1429, 1504)] * 8,
        [(1462, 1359)] * 8, [(2890, 454)] * 2, [(7203, 325)], [(4168, 522)] * 3,
        [(4273, 649)] * 4, [(3898, 963)] * 3, [(1104, 7692)], [(2304, 4096)],
        [(1500, 1024), (33, 500), (1024, 1024), (1000, 2048)] * 2]


@pytest.mark.parametrize("products", [1, 3])
@pytest.mark.parametrize("shapes", SETS, ids=lambda s: f"{len(s)}of{s[0][0]}x{s[0][1]}")
def test_every_tile(shapes, products):
    xs = [matrix(*s, seed=i) for i, s in enumerate(shapes)]
    ys = orth(xs, products)
    for i in {0, len(xs) // 2, len(xs) - 1} if len(set(shapes)) == 1 else range(len(xs)):
        assert off(ys[i], ns64(xs[i])) <= BAR[products], i


def test_views_of_a_flat_buffer():
    """Matrices that start at any element (no 16-byte accesses): the same bits as
    aligned copies, and nothing else written."""
    shapes = [(77, 90), (64, 72), (33, 41)]
    d = F.muon_descs(shapes)
    ws = F.workspace(F.fp16_muon_workspace_bytes(d, 1))
    bufs = []
    for k, scale in ((1, 0.1), (2, 1e-3), (3, 1e-3)):
        flat = torch.full((1 + sum(a * b for a, b in shapes) + 9,), 7.0, dtype=torch.float16,
                          device="cuda")
        views, at = [], 1
        for i, s in enumerate(shapes):
            v = flat[at:at + s[0] * s[1]].view(s)
            v.copy_(matrix(*s, seed=10 * k + i, kind="normal", scale=scale))
            views.append(v)
            at += s[0] * s[1]
        bufs.append((flat, views, at))
    copies = [[v.clone() for v in views] for _, views, _ in bufs]
    run = lambda l: F.fp16_muon_step(d, l[0], l[1], l[2], 0.02, 0.9, 0.1, ws=ws)
    note("[gpu] muon on views")
    run([b[1] for b in bufs])
    run(copies)
    torch.cuda.synchronize()
    for (flat, views, at), cs in zip(bufs, copies):
        assert all(torch.equal(v, c) for v, c in zip(views, cs))
        assert flat[0] == 7 and (flat[at:] == 7).all()


@pytest.mark.parametrize("products", [1, 3])
def test_many_matrices_at_once_as_one_by_one(products):
    """1024 small matrices and a large one among them; each within the bar."""
    shapes = [(1 + (7 * i) % 40, 1 + (13 * i) % 50) for i in range(1023)] + [(200, 300)]
    xs = [matrix(*s, seed=i, kind="normal") for i, s in enumerate(shapes)]
    ys = orth(xs, products)
    for i, (x, y) in enumerate(zip(xs, ys)):
        if i % 31 == 0 or i >= 1020:
            assert off(y, ns64(x)) <= BAR[products], shapes[i]
        assert torch.isfinite(y).all(), shapes[i]


@pytest.mark.parametrize("shape", [(100, 160), (50, 90)], ids=["tiles", "workgroup"])
def test_steps_and_coefficients(shape):
    x = matrix(*shape, 3)
    cubic = [(1.5, -0.5, 0.0)] * 8
    mixed = [(3.0, -3.2, 1.2), (2.5, -2.0, 0.5), (1.875, -1.25, 0.375)]
    for steps, coef in [(1, None), (2, QUINTIC), (8, cubic), (3, mixed)]:
        y, = orth([x], 3, steps, coef)
        assert off(y, ns64(x, steps, coef)) <= BAR[3], (steps, coef)


@pytest.mark.parametrize("shape", [(70, 80), (48, 80)], ids=["tiles", "workgroup"])
def test_scale_and_size_of_the_input(shape):
    """The result does not depend on the input's size, down to subnormal entries."""
    for scale in (3e4, 1.0, 2.0 ** -20):
        x = matrix(*shape, 5, "normal", scale)
        x = x.clamp(-65504, 65504)
        y, = orth([x], 3, scales=[0.25])
        assert off(y, ns64(x, scale=0.25)) <= BAR[3], scale
    one = torch.zeros((shape[0] - 45, 5), dtype=torch.float16)
    one[1, 2] = 2.0 ** -24
    y, = orth([one], 3)
    assert off(y, ns64(one)) <= BAR[3]


@pytest.mark.parametrize("shape", [(70, 90), (60, 91)], ids=["tiles", "workgroup"])
def test_zero_and_not_finite(shape):
    z = torch.zeros(shape, dtype=torch.float16)
    rows = matrix(*shape, 1)
    rows[10:50] = 0
    cols = matrix(*shape, 2)
    cols[:, 3:] = 0
    nan, inf = matrix(*shape, 3), matrix(*shape, 4)
    nan[4, 5] = float("nan")
    inf[-1, -1] = float("-inf")
    for products in (1, 3):
        y = orth([z, rows, nan, cols, inf, rows], products)
        assert (y[0] == 0).all()
        assert (y[1][10:50] == 0).all() and off(y[1], ns64(rows)) <= BAR[products]
        assert (y[3][:, 3:] == 0).all() and off(y[3], ns64(cols)) <= BAR[products]
        assert torch.isnan(y[2]).all() and torch.isnan(y[4]).all()
        assert torch.equal(y[5], y[1])


@pytest.mark.parametrize("shape", [(137, 141), (37, 41)], ids=["tiles", "workgroup"])
def test_in_place_and_nothing_else_written(shape):
    x = matrix(*shape, 7)
    ref = ns64(x)
    n = x.numel()
    buf = torch.full((n + 64,), 3.0, dtype=torch.float16, device="cuda")
    v = buf[8:8 + n].view(shape)
    v.copy_(x)
    d = F.muon_descs([shape])
    need = F.fp16_muon_workspace_bytes(d, 3)
    ws = torch.full((need + 256,), 0xA5, dtype=torch.uint8, device="cuda")
    F.fp16_orthogonalize(d, [v], [v], products=3, ws=ws, ws_bytes=need)
    torch.cuda.synchronize()
    assert off(v, ref) <= BAR[3]
    assert (buf[:8] == 3).all() and (buf[8 + n:] == 3).all() and (ws[need:] == 0xA5).all()


@pytest.mark.parametrize("rows", [300, 30], ids=["tiles", "workgroup"])
def test_same_bits_again_and_on_another_stream(rows):
    xs = [matrix(rows, 200, 1), matrix(64, 576, 2)]
    a, b = orth(xs, 1), orth(xs, 1)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        c = orth(xs, 1)
    for x, y, z in zip(a, b, c):
        assert torch.equal(x, y) and torch.equal(x, z)


@pytest.mark.parametrize("products", [1, 3])
@pytest.mark.parametrize("shape", [(16300, 65500), (65500, 16300)], ids=["wide", "tall"])
def test_the_largest_matrices(shape, products):
    """Offsets past 2^31 bytes.  One element a row and column of the shorter side, so
    that the singular values are known, every product of two rows is zero, and the
    result is the polynomial of each element on its own; everything else stays zero."""
    require_gpu()
    m, n = min(shape), max(shape)
    v = (1.0 + 0.5 * torch.sin(torch.arange(m, dtype=torch.float64))).half()
    i = torch.arange(m, device="cuda")
    j = n - 1 - 4 * i  # to the far end of the last row
    at = i * n + j if shape[0] == m else j * m + i
    x = torch.zeros(shape, dtype=torch.float16, device="cuda")
    x.view(-1)[at] = v.cuda()
    d = F.muon_descs([(*shape, 1.0)])
    ws = F.workspace(F.fp16_muon_workspace_bytes(d, products))
    note(f"[gpu] orthogonalize {shape} products={products}")
    F.fp16_orthogonalize(d, [x], [x], 2, None, products, ws)
    torch.cuda.synchronize()
    s = v.double() / v.double().norm()
    for _ in range(2):
        s = QUINTIC[0] * s + QUINTIC[1] * s ** 3 + QUINTIC[2] * s ** 5
    got = x.view(-1)[at]
    assert off(got, s.cuda()) <= BAR[products]
    x.view(-1)[at] = 0
    assert not x.view(torch.int16).any()


# ---- the update --------------------------------------------------------------------

def step(ws_, gs, ms, scales, lr, mu, wd, nesterov, products, steps=5):
    require_gpu()
    d = F.muon_descs([(w.shape[0], w.shape[1], s) for w, s in zip(ws_, scales)])
    work = F.workspace(F.fp16_muon_workspace_bytes(d, products))
    note(f"[gpu] muon {[tuple(w.shape) for w in ws_][:6]} products={products}")
    F.fp16_muon_step(d, ws_, gs, ms, lr, mu, wd, nesterov, steps, None, products, work)
    torch.cuda.synchronize()


@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("products", [1, 3])
def test_update(products, nesterov):
    """Momentum bit for bit; the weights from the float64 direction: the update's
    relative error as above, one rounding of w and float32's of the rest."""
    shapes, scales = [(64, 147), (200, 72), (33, 130)], [1.0, 1.5, 0.7]
    lr, mu, wd = 0.02, 0.95, 0.1
    g = [matrix(*s, seed=10 + i) for i, s in enumerate(shapes)]
    m = [matrix(*s, seed=20 + i) for i, s in enumerate(shapes)]
    w = [matrix(*s, seed=30 + i, kind="normal", scale=0.1) for i, s in enumerate(shapes)]
    W, G, M = ([t.cuda() for t in l] for l in (w, g, m))
    for _ in range(2):  # the second update starts from the first's results
        w0, m0 = [t.cpu() for t in W], [t.cpu() for t in M]
        step(W, G, M, scales, lr, mu, wd, nesterov, products)
        for i in range(len(shapes)):
            _, mr = oracle.sgd_f32(np.zeros(g[i].numel(), np.float16), g[i].numpy().ravel(),
                                   m0[i].numpy().ravel(), 0.1, mu, 0.0)
            assert np.array_equal(host(M[i]).ravel().view(np.uint16), mr.view(np.uint16))
            md = torch.from_numpy(mr).view(*shapes[i]).double()
            o = ns64(g[i].double() + float(np.float32(mu)) * md if nesterov else md)
            upd = lr * scales[i] * o
            ref = (1 - lr * wd) * w0[i].double().cuda() - upd
            err = (W[i].double() - ref).norm().item()
            bar = BAR[products] * upd.norm().item() + (2.0 ** -11 + 2.0 ** -20) * ref.norm().item()
            assert err <= bar + 2.0 ** -25 * math.sqrt(ref.numel())


@pytest.mark.parametrize("products", [1, 3])
def test_update_of_small_matrices(products):
    """The same on one workgroup each, views of odd alignment with borders, and the
    momentum and weights beside them left alone."""
    shapes = [(64, 147), (147, 64), (5, 3), (64, 1024), (1024, 64), (33, 1000), (1000, 33), (1, 9)]
    assert F.fp16_muon_kernels(F.muon_descs(shapes), products) == "one workgroup each"
    lr, mu, wd = 0.02, 0.95, 0.1

    def place(l):
        out = []
        for i, t in enumerate(l):
            flat = torch.full((t.numel() + 40,), 7.0, dtype=torch.float16, device="cuda")
            v = flat[1 + i:1 + i + t.numel()].view(t.shape)
            v.copy_(t)
            out.append((flat, v))
        return [f for f, _ in out], [v for _, v in out]

    g = [matrix(*s, seed=10 + i) for i, s in enumerate(shapes)]
    m = [matrix(*s, seed=20 + i) for i, s in enumerate(shapes)]
    w = [matrix(*s, seed=30 + i, kind="normal", scale=0.1) for i, s in enumerate(shapes)]
    (GF, G), (MF, M), (WF, W) = place(g), place(m), place(w)
    step(W, G, M, [1.0] * len(shapes), lr, mu, wd, True, products)
    for i, s in enumerate(shapes):
        _, mr = oracle.sgd_f32(np.zeros(g[i].numel(), np.float16), g[i].numpy().ravel(),
                               m[i].numpy().ravel(), 0.1, mu, 0.0)
        assert np.array_equal(host(M[i]).ravel().view(np.uint16), mr.view(np.uint16))
        upd = lr * ns64(g[i].double() + float(np.float32(mu)) * torch.from_numpy(mr).view(*s).double())
        ref = (1 - lr * wd) * w[i].double().cuda() - upd
        bar = BAR[products] * upd.norm().item() + (2.0 ** -11 + 2.0 ** -20) * ref.norm().item()
        assert (W[i].double() - ref).norm().item() <= bar + 2.0 ** -25 * math.sqrt(ref.numel()), s
        assert torch.equal(G[i].cpu(), g[i])
        for f in (GF[i], MF[i], WF[i]):
            assert (f[:1 + i] == 7).all() and (f[1 + i + g[i].numel():] == 7).all()


def test_update_alone():
    """From zero weights, without decay: w = -lr scale O, held to O's bar."""
    for shape in [(64, 576), (300, 520), (1000, 257)]:
        g = matrix(*shape, seed=4)
        W, M = (torch.zeros(shape, dtype=torch.float16, device="cuda") for _ in range(2))
        step([W], [g.cuda()], [M], [2.0], 0.5, 0.9, 0.0, True, 1)
        assert torch.equal(M.cpu(), g)
        assert off(W, -ns64(g)) <= BAR[1]


@pytest.mark.parametrize("wide", [128, 60], ids=["tiles", "workgroup"])
def test_update_in_a_graph(wide):
    """Captured once, replayed with eager work between the replays: each replay as
    the eager update from the same state."""
    require_gpu()
    shapes = [(64, 147), (256, wide), (40, 700)]
    d = F.muon_descs([(*s, 1.0) for s in shapes])
    mk = lambda o, sc: [matrix(*s, seed=o + i, scale=sc).cuda() for i, s in enumerate(shapes)]
    W, G, M = mk(1, 0.1), mk(2, 1e-3), mk(3, 1e-3)
    ws = F.workspace(F.fp16_muon_workspace_bytes(d, 1))
    We, Me = [t.clone() for t in W], [t.clone() for t in M]
    run = lambda a, b: F.fp16_muon_step(d, a, G, b, 0.02, 0.95, 0.01, ws=ws)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        run([t.clone() for t in W], [t.clone() for t in M])
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(W, M)
    for i in range(4):
        G[i % 3].mul_(1.5)
        graph.replay()
        torch.cuda.synchronize()
        run(We, Me)
        torch.cuda.synchronize()
        for a, b in zip(W + M, We + Me):
            assert torch.equal(a, b), i
