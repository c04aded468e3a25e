"""The dense head's operators together, as a program runs them: a block of two dense layers
on a residual stream, dropout, a classifier, log probabilities with entropies and their
gradients all the way back, eagerly, captured in a graph beside another program's, and on a
stream of its own."""

import numpy as np
import pytest
import torch

import head_oracle as O
import paper_1911_07384_amd as F
from gpu_util import dev, host, note, require_gpu

pytestmark = pytest.mark.gpu


def half(r, *s, std=1.0):
    return (std * r.standard_normal(s)).astype(np.float16)


class Program:
    """tokens rows of `width`: x + drop(W2 gelu-layer(x)), dropout, classifier, loss."""

    P = 0.2

    def __init__(self, tokens, width, inner, classes, seed, stream=None):
        require_gpu()
        r = np.random.default_rng(seed)
        self.n, self.k = tokens, classes
        self.host = {"x": half(r, tokens, width), "w1": half(r, inner, width, std=width ** -0.5),
                     "b1": half(r, inner, std=0.2), "w2": half(r, width, inner, std=inner ** -0.5),
                     "b2": half(r, width, std=0.2), "w3": half(r, classes, width, std=width ** -0.5),
                     "b3": half(r, classes, std=0.2)}
        self.tok = r.integers(0, classes, tokens).astype(np.int32)
        self.tok[::5] = -1
        self.seed = seed
        g = {k: dev(v) for k, v in self.host.items()}
        self.g, self.t = g, torch.from_numpy(self.tok).cuda()
        self.d1 = F.dense_desc(tokens, width, inner, "gelu")
        self.d2 = F.dense_desc(tokens, inner, width, "none", self.P, 1)
        self.d3 = F.dense_desc(tokens, width, classes)
        self.lp = F.logprob_desc(tokens, classes, top=3, scale=1.5)
        self.rng = F.rng_state(seed, 0)
        self.ws = F.workspace(max([F.fp16_dense_workspace_bytes(d) for d in
                                   (self.d1, self.d2, self.d3)]
                                  + [F.fp16_logprobs_workspace_bytes(self.lp)]))
        e = lambda *s: torch.zeros(s, dtype=torch.float16, device="cuda")
        f = lambda *s: torch.zeros(s, dtype=torch.float32, device="cuda")
        o = self.o = {"z1": e(tokens, inner), "a1": e(tokens, inner), "y": e(tokens, width),
                      "yd": e(tokens, width), "z": e(tokens, classes), "logp": f(tokens),
                      "stats": f(tokens, 3), "top_id": f(tokens, 3).int(), "top_logp": f(tokens, 3),
                      "dz": e(tokens, classes), "dyd": e(tokens, width), "dy": e(tokens, width),
                      "da1": e(tokens, inner), "dx": e(tokens, width)}
        for k in ("w1", "b1", "w2", "b2", "w3", "b3"):
            o["d" + k] = torch.zeros_like(g[k])
        self.dlogp, self.dent = f(tokens) - 1.0 / tokens, f(tokens) - 0.01 / tokens

    def step(self, stream=None):
        g, o, ws, kw = self.g, self.o, self.ws, dict(rng=self.rng, ws=self.ws, stream=stream)
        F.fp16_dense_fwd(self.d1, g["x"], g["w1"], g["b1"], None, o["a1"], o["z1"], **kw)
        F.fp16_dense_fwd(self.d2, o["a1"], g["w2"], g["b2"], g["x"], o["y"], **kw)
        F.fp16_dropout(o["y"], None, o["yd"], self.P, self.rng, 2, stream=stream)
        F.fp16_dense_fwd(self.d3, o["yd"], g["w3"], g["b3"], None, o["z"], **kw)
        F.fp16_logprobs(self.lp, o["z"], self.t, o["logp"], o["stats"], o["top_id"],
                        o["top_logp"], ws=ws, stream=stream)
        F.fp16_logprobs_bwd(self.lp, o["z"], self.t, o["stats"], self.dlogp, self.dent, o["dz"],
                            stream=stream)
        F.fp16_dense_bwd(self.d3, o["yd"], g["w3"], None, o["dz"], o["dyd"], o["dw3"], o["db3"], **kw)
        F.fp16_dropout(o["dyd"], None, o["dy"], self.P, self.rng, 2, stream=stream)
        F.fp16_dense_bwd(self.d2, o["a1"], g["w2"], None, o["dy"], o["da1"], o["dw2"], o["db2"], **kw)
        # the block's input: its own gradient and the residual stream's
        F.fp16_dense_bwd(self.d1, g["x"], g["w1"], o["z1"], o["da1"], o["dx"], o["dw1"], o["db1"],
                         **kw)
        F.fp16_dropout(o["dx"], o["dy"], o["dx"], 0.0, self.rng, 0, stream=stream)
        F.fp16_rng_advance(self.rng, stream=stream)

    def results(self):
        return {k: host(v).copy() for k, v in self.o.items()}

    def check(self, step):
        """Every result against 64 bits from its own inputs, then the whole way back
        against autograd in 64 bits."""
        h, r = self.host, self.results()
        rng = (self.seed, step)
        D = lambda *a, **k: O.Dense(*a, **k)
        one = D(h["x"], h["w1"], h["b1"], act="gelu", z=r["z1"], dy=r["da1"])
        two = D(r["a1"], h["w2"], h["b2"], h["x"], p=self.P, rng=rng, site=1, dy=r["dy"])
        three = D(r["yd"], h["w3"], h["b3"], dy=r["dz"])
        for got, w, err, what in [
                ("a1", one.y, one.y_err, 1), ("z1", one.z, one.z_err, 1), ("y", two.y, two.y_err, 2),
                ("z", three.y, three.y_err, 3), ("dyd", three.dx, three.dx_err, 3),
                ("dw3", three.dw, three.dw_err, 3), ("db3", three.db, three.db_err, 3),
                ("da1", two.dx, two.dx_err, 2), ("dw2", two.dw, two.dw_err, 2),
                ("db2", two.db, two.db_err, 2), ("dw1", one.dw, one.dw_err, 1),
                ("db1", one.db, one.db_err, 1)]:
            O.close(r[got], w, err, f"{got} of layer {what}")
        assert np.array_equal(r["yd"], O.dropout(r["y"], None, self.P, *rng, 2))
        assert np.array_equal(r["dy"], O.dropout(r["dyd"], None, self.P, *rng, 2))
        L = O.Logprob(r["z"], 1.5, 3)
        assert np.array_equal(r["top_id"], L.top_id)
        # autograd
        T = {k: O.t64(v).requires_grad_() for k, v in h.items()}
        keep = lambda s, site, shape: (torch.from_numpy(O.kept(int(np.prod(shape)), self.P, *rng, site))
                                       .view(shape) * float(O.factor(self.P)))
        a1 = O.activate(T["x"] @ T["w1"].T + T["b1"], "gelu")
        y = (a1 @ T["w2"].T + T["b2"]) * keep(1, 1, (self.n, T["x"].shape[1])) + T["x"]
        z = (y * keep(2, 2, y.shape)) @ T["w3"].T + T["b3"]
        lp = torch.log_softmax(1.5 * z, 1)
        asked = torch.from_numpy(self.tok) >= 0
        at = torch.from_numpy(self.tok).long().clamp(min=0)[:, None]
        ent = -(lp.exp() * lp).sum(1)
        loss = -(lp.gather(1, at)[:, 0][asked].sum() + 0.01 * ent.sum()) / self.n
        loss.backward()
        for k in ("x", "w1", "b1", "w2", "b2", "w3", "b3"):
            g, want = torch.from_numpy(r["d" + k]).double(), T[k].grad
            # some ten roundings to binary16 in a row, each 2^-11 of its values, and their
            # smallest step on gradients of about 1e-3 / n
            tiny = 40 * O.TINY * want.numel() ** 0.5
            assert (g - want).norm() <= 16 * O.HALF * want.norm() + tiny, k


SIZES = [(40, 96, 200, 300), (7, 33, 65, 1001), (300, 256, 520, 1000)]


@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_together(size):
    p = Program(*size, seed=sum(size))
    note(f"[gpu] head {size}")
    for step in range(2):
        p.step()
        torch.cuda.synchronize()
        p.check(step)


def test_on_another_stream_and_in_graphs_of_two_programs():
    """Two programs with workspaces of their own, each captured once, replayed in turn and
    on two streams at once; every replay equals the eager steps, bit for bit."""
    a, b = Program(*SIZES[0], seed=1), Program(*SIZES[2], seed=2)
    want = []
    for p in (a, b):
        rows = []
        for _ in range(4):
            p.step()
            torch.cuda.synchronize()
            rows.append(p.results())
        want.append(rows)
        p.rng.copy_(F.rng_state(p.seed, 0))
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    a.step(stream=s)  # on a stream that is not torch's current one
    s.synchronize()
    got = a.results()
    assert all(np.array_equal(got[k], want[0][0][k], equal_nan=True) for k in got)
    a.rng.copy_(F.rng_state(a.seed, 0))
    graphs = []
    for p in (a, b):
        note("[gpu] capture of a head")
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            p.step()
        p.rng.copy_(F.rng_state(p.seed, 0))
        graphs.append(g)
    torch.cuda.synchronize()
    for i in range(4):
        if i < 2:
            for g in graphs:
                g.replay()
        else:
            with torch.cuda.stream(s):
                graphs[0].replay()
            graphs[1].replay()
        torch.cuda.synchronize()
        assert np.isfinite((torch.randn(1000, device="cuda") * 2).sum().item())  # eager work
        for p, rows in zip((a, b), want):
            got = p.results()
            assert all(np.array_equal(got[k], rows[i][k], equal_nan=True) for k in got), i


def test_large_offsets():
    """A matrix past 2^31 elements on each side of the product: the last rows of y and of
    dW, and the rows of x behind 4 GB."""
    require_gpu()
    t, i, o = 16, (1 << 20) - 8, 2056  # W 2.16e9 elements
    note("[gpu] dense with 2^31 weights")
    w = torch.zeros((o, i), dtype=torch.float16, device="cuda")
    x = torch.zeros((t, i), dtype=torch.float16, device="cuda")
    x[:, -1], x[:, 0] = torch.arange(t).cuda().half(), 1.0
    w[:, -1], w[:, 0] = (torch.arange(o) % 7).cuda().half(), 0.5
    d = F.dense_desc(t, i, o)
    y = torch.empty((t, o), dtype=torch.float16, device="cuda")
    ws = F.workspace(F.fp16_dense_workspace_bytes(d))
    F.fp16_dense_fwd(d, x, w, None, None, y, ws=ws)
    torch.cuda.synchronize()
    want = torch.arange(t)[:, None] * (torch.arange(o) % 7)[None, :] + 0.5
    assert torch.equal(y.cpu().double(), want.double())
    dy = torch.zeros_like(y)
    dy[3, -1], dy[5, 0] = 2.0, 1.0
    dx = torch.empty_like(x)
    dw = torch.empty_like(w)
    F.fp16_dense_bwd(d, x, w, None, dy, dx, dw, ws=ws)
    torch.cuda.synchronize()
    assert torch.equal(dx[3], 2.0 * w[-1]) and torch.equal(dx[5], w[0])
    assert torch.equal(dw[-1], 2.0 * x[3]) and torch.equal(dw[0], x[5]) and not dw[1:-1].any()
    del dw
    # the same with many rows of y: tokens x outputs past 2^31
    t, i, o = 1 << 20, 64, 2056
    note("[gpu] dense with 2^31 outputs")
    x = torch.zeros((t, i), dtype=torch.float16, device="cuda")
    x[:, 0] = (torch.arange(t) % 61).cuda().half()
    w = torch.zeros((o, i), dtype=torch.float16, device="cuda")
    w[:, 0] = (torch.arange(o) % 31).cuda().half()
    d = F.dense_desc(t, i, o, "relu")
    y = torch.empty((t, o), dtype=torch.float16, device="cuda")
    F.fp16_dense_fwd(d, x, w, None, None, y, ws=F.workspace(F.fp16_dense_workspace_bytes(d, 0)))
    torch.cuda.synchronize()
    for r in (0, 1 << 19, (1 << 20) - 1, (1 << 20) - 300):
        assert torch.equal(y[r].cpu().double(), (r % 61) * (torch.arange(o) % 31).double())
    # its gradients: dz = y's slope times ones
    dy = torch.ones_like(y)
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    db = torch.empty(o, dtype=torch.float16, device="cuda")
    z = y
    F.fp16_dense_bwd(d, x, w, z, dy, dx, dw, db, ws=F.workspace(F.fp16_dense_workspace_bytes(d, 1)))
    torch.cuda.synchronize()
    on = torch.arange(o) % 31 != 0
    total = float(((torch.arange(o) % 31)[on]).sum())
    for r in (1, (1 << 20) - 1):
        got = dx[r, 0].item()
        assert got == torch.tensor(total if r % 61 else 0.0).half().item()
    count = float((torch.arange(t) % 61 != 0).sum())
    assert torch.isinf(db[on.cuda()]).all() and count > 65504 and not db[~on.cuda()].any()
