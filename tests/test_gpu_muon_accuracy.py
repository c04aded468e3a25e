"""How exact the orthogonalised direction O is, below the rounding of what holds it.

fp16_muon_step from w0 = rne16(O64) (O64 the direction in float64, brought to entries
near 1 by a power of two in lr), without momentum or decay, gives w = rne16(w0 - O):
the difference is about 2^-12 of O, so w0 - w is O to about 2^-22 of it.

Bars, relative in the 2-norm, of five steps of the default coefficients, with
p(s) = as + bs^3 + cs^5 and u = 2^-11 (products = 1) or 2^-22 (3), the roundings of an
operand's entries relative to them:

RANDOM matrices, whose entries round independently.  Near s = 1 a step adds |B| = 2.7 of
X's rounding and |bs^2 + 2cs^4| <= 1.4 of A's, sqrt(2) of X's.  The rounding is
u / sqrt(3) at most and 0.41 u in the mean over a binade (rms), so (2.7^2 + 2^2)^(1/2) *
0.41 u = 1.4 u a step, and |p'| = 1.14, 1.29, 1.26, 0.74 on the orbit from 1 make
(1 + 0.55 + 0.87 + 1.44 + 1.88)^(1/2) * 1.4 u = 3.3 u of five: 1.6e-3.  Half as much
again for singular values off that orbit: 2.5e-3.  That takes roundings to average, in
the entries of 16 rows and columns at least.  One row or column has a single singular
value, whose errors of 3 |bs^2 + 2cs^4| + 2 |B| roundings all add: the bar of the
coherent ones below, for shorter sides under 16.  With products = 3 float32 sums of L terms
add 0.3 * 2^-23 * (L / 3)^(1/2) a step, 6e-7 for L = 3 * 8192 / 16, in place of 1.4 u =
3.3e-7: five give 1.6e-6 by the same factors; 1e-5 holds that six times over, and fails
with operands of 18 bits.  An element's own rounding is proportional to it: elementwise
8 bars of the rms plus 8 u of the element.

COHERENT matrices (rank one, equal rows, all entries of one magnitude): roundings may
all be of one sign.  A step adds at most
  c(s) u = s (3 |bs^2 + 2cs^4| + 2 |bs^2 + cs^4|) u
(X's rounding twice and A's in A; B's and X's in BX) and multiplies what is there by
|p'| along the singular vectors or p(s) / s across them: the recurrence `coherent`, run
over the whole interval that the error allows.  With products = 3 rounding errors in
the directions of zero singular values, orthogonal to all of X, grow 3.4445 times a
step: 0.3 * 2^-23 * (L / 3)^(1/2) * 2.8 of each step's sums, L = 3 * 2500 / 16, times
(3.4445^5 - 1) / (2.4445 * 0.7) makes 2.4e-4: 3e-4 for shorter sides up to 2500.
"""

import math

import numpy as np
import pytest
import torch

import paper_1911_07384_amd as F
from gpu_util import note, require_gpu
from test_gpu_muon import QUINTIC, SETS, SHAPES, matrix, ns64

pytestmark = pytest.mark.gpu

U = {1: 2.0 ** -11, 3: 2.0 ** -22}
LOW_RANK = 3e-4


def poly(s):
    a, b, c = QUINTIC
    return a * s + b * s ** 3 + c * s ** 5


def coherent(steps, u):
    """The relative error that `steps` steps from s = 1 may reach."""
    a, b, c = QUINTIC
    s, e = 1.0, 0.0
    for _ in range(steps):
        d = np.linspace(s - e, s + e, 401)
        local = d * (3 * abs(b * d ** 2 + 2 * c * d ** 4) + 2 * abs(b * d ** 2 + c * d ** 4)) * u
        e = max(abs(poly(d) - poly(s)).max(), e * (poly(d) / d).max()) + local.max()
        s = poly(s)
    return e / s


def random_bar(shape, products):
    bar = {1: 2.5e-3, 3: 1e-5}[products]
    return bar if min(shape) >= 16 else max(bar, coherent(5, U[products]))


def directions(xs, refs, products, steps=5):
    """O of every matrix of a set, in float64."""
    require_gpu()
    rms = torch.stack([r.square().mean() for r in refs]).max().sqrt().item()
    lr = 2.0 ** round(-math.log2(rms))
    W = [(lr * r).half().contiguous() for r in refs]
    W0 = [w.double() for w in W]
    d = F.muon_descs([tuple(x.shape) for x in xs])
    ws = F.workspace(F.fp16_muon_workspace_bytes(d, products))
    note(f"[gpu] direction {[tuple(x.shape) for x in xs][:6]} products={products} steps={steps}")
    F.fp16_muon_step(d, W, [x.cuda() for x in xs], [torch.zeros_like(w) for w in W], lr, 0.0, 0.0,
                     False, steps, None, products, ws)
    torch.cuda.synchronize()
    return [(a - b.double()) / lr for a, b in zip(W0, W)]


def orthogonalised(xs, products):
    d = F.muon_descs([tuple(x.shape) for x in xs])
    X = [x.cuda() for x in xs]
    Y = [torch.full_like(x, float("nan")) for x in X]
    F.fp16_orthogonalize(d, X, Y, products=products, ws=F.workspace(
        F.fp16_muon_workspace_bytes(d, products)))
    torch.cuda.synchronize()
    return Y


def check_elements(got, ref, products, rounded):
    """Every element of O (or of y, rounded once more)."""
    rms = ref.square().mean().sqrt()
    tol = 8 * random_bar(ref.shape, products) * rms + 8 * U[products] * ref.abs()
    if rounded:
        tol = tol * (1 + 2.0 ** -11) + 2.0 ** -11 * ref.abs() + 2.0 ** -25
    wrong = (~((got.double() - ref).abs() <= tol)).nonzero()
    assert len(wrong) == 0, (len(wrong), wrong[:8].tolist())


@pytest.mark.parametrize("products", [1, 3])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"{s[0]}x{s[1]}")
@pytest.mark.parametrize("kind", ["noisy", "normal"])
def test_every_element(kind, shape, products):
    x = matrix(*shape, seed=sum(shape) + 1, kind=kind)
    ref = ns64(x)
    o, = directions([x], [ref], products)
    assert (o - ref).norm() <= random_bar(ref.shape, products) * ref.norm()
    check_elements(o, ref, products, False)
    check_elements(orthogonalised([x], products)[0], ref, products, True)


@pytest.mark.parametrize("products", [1, 3])
@pytest.mark.parametrize("shapes", SETS, ids=lambda s: f"{len(s)}of{s[0][0]}x{s[0][1]}")
def test_every_element_of_every_matrix_of_a_set(shapes, products):
    """On every tile that the products run on (see SETS)."""
    xs = [matrix(*s, seed=100 + i) for i, s in enumerate(shapes)]
    refs = [ns64(x) for x in xs]
    os_, ys = directions(xs, refs, products), orthogonalised(xs, products)
    for i, (o, y, ref) in enumerate(zip(os_, ys, refs)):
        assert (o - ref).norm() <= random_bar(ref.shape, products) * ref.norm(), i
        check_elements(o, ref, products, False)
        check_elements(y, ref, products, True)


COHERENT = [(2, 2), (3, 3), (8, 8), (17, 64), (64, 64), (89, 92), (110, 110), (64, 576), (576, 64),
            (333, 1111), (1000, 2048), (64, 16384), (1500, 1500)]


def coherent_matrix(kind, m, n):
    g = torch.Generator().manual_seed(3 + m + n)
    sign = lambda *s: 1.0 - 2.0 * torch.randint(0, 2, s, generator=g)
    normal = lambda *s: torch.randn(s, generator=g)
    x = {"constant": lambda: torch.full((m, n), 0.0137), "signs": lambda: sign(m, 1) * sign(1, n),
         "rows": lambda: normal(1, n).expand(m, n), "columns": lambda: normal(m, 1).expand(m, n),
         "outer": lambda: torch.randint(-7, 8, (m, 1), generator=g) * normal(1, n),
         "two": lambda: normal(2, n)[torch.arange(m) % 2], "plus_minus": lambda: sign(m, n),
         "identity": lambda: torch.eye(m, n)}[kind]()
    return x.half().contiguous()


@pytest.mark.parametrize("products", [1, 3])
@pytest.mark.parametrize("kind", ["constant", "signs", "rows", "columns", "outer", "two",
                                  "plus_minus", "identity"])
def test_entries_that_round_alike(kind, products):
    for shape in COHERENT:
        x = coherent_matrix(kind, *shape)
        if not x.any():
            continue
        for steps in (1, 3, 5):
            ref = ns64(x, steps)
            o, = directions([x], [ref], products, steps)
            off = ((o - ref).norm() / ref.norm()).item()
            bar = coherent(steps, U[1]) if products == 1 else LOW_RANK
            assert off <= bar, (shape, steps, off)


@pytest.mark.parametrize("products", [1, 3])
def test_more_steps_of_low_rank(products):
    """Past five steps the errors of zero singular values go on growing by 3.4445."""
    for kind in ("rows", "outer"):
        x = coherent_matrix(kind, 200, 300)
        ref = ns64(x, 8)
        o, = directions([x], [ref], products, 8)
        bar = {1: coherent(8, U[1]), 3: LOW_RANK * QUINTIC[0] ** 3}[products]
        assert (o - ref).norm() <= bar * ref.norm()
