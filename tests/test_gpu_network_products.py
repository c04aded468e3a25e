"""The training step with the operators beside the convolutions, as a program runs
them together, on the GPU:

1. ResNet-50 with its classifier in 8-bit integers and its weights updated by
   orthogonalised momentum: the new calls replayed on the inputs that the GPU's saw
   (the classifier's products bit for bit, the update at the bars of test_gpu_muon),
   graph replays equal to eager steps, and everything before the classifier as in
   the plain network.
2. One dense layer trained for some steps (quantise, forward, backward, update),
   every step's results checked, captured into a graph with a second program of its
   own stream and workspace beside it.
"""

import numpy as np
import pytest
import torch

import oracle
import paper_1911_07384_amd as F
from gpu_util import host, note, require_gpu
from paper_1911_07384_amd.network import ResNet50
from test_gpu_int8 import acts, gpu, product, quant_rows, same
from test_gpu_muon import BAR, ns64

pytestmark = pytest.mark.gpu


def _net(**kw):
    require_gpu()
    net = ResNet50(n=4, image=64, seed=3, **kw)
    net.load_batch(3)
    return net


def check_update(w0, g, m0, w1, m1, scale, lr, mu, wd, products):
    """One update's momentum bit for bit and its weights within the direction's bar."""
    _, mr = oracle.sgd_f32(np.zeros(g.size, np.float16), g.ravel(), m0.ravel(), 0.1, mu, 0.0)
    assert np.array_equal(m1.ravel().view(np.uint16), mr.view(np.uint16))
    md = torch.from_numpy(mr.reshape(g.shape)).double()
    upd = lr * scale * ns64(torch.from_numpy(g).double() + float(np.float32(mu)) * md)
    ref = (1 - lr * wd) * torch.from_numpy(w0).double().cuda() - upd
    err = (torch.from_numpy(w1).double().cuda() - ref).norm().item()
    assert err <= (BAR[products] * upd.norm().item() + (2.0 ** -11 + 2.0 ** -20) * ref.norm().item()
                   + 2.0 ** -25 * ref.numel() ** 0.5)


def test_network_calls():
    net, plain = _net(optimizer="muon", classifier="int8"), _net()
    note("[gpu] ResNet-50 step with muon and the 8-bit classifier")
    b = net.buffers
    muon = net.upd[0].a
    w0 = [host(t).copy() for t in muon["w"]]
    m0 = [host(t).copy() for t in muon["m"]]
    net.forward()
    plain.forward()
    torch.cuda.synchronize()
    # the same network up to the classifier
    assert torch.equal(b["gap.y"], plain.buffers["gap.y"])
    x, w = host(b["gap.y"]).reshape(4, -1), host(b["fc"]).reshape(1000, -1)
    y = host(b["fc.y"]).reshape(4, -1)
    assert same(y, product(*quant_rows(x), *quant_rows(w)))
    # ... and close to the product of the unquantised operands: each operand is off by
    # at most half a step of max / 127 an element, 2048 independent terms; 8 standard
    # deviations of that (uniform, 1/12 of a step squared) plus the rounding
    step = lambda a: np.abs(a).max(1, keepdims=True).astype(np.float64) / 127
    sd = np.sqrt(((step(x) ** 2 / 12) * (w.astype(np.float64) ** 2).sum(1)[None, :])
                 + (x.astype(np.float64) ** 2).sum(1)[:, None] * (step(w).T ** 2 / 12))
    exact = x.astype(np.float64) @ w.astype(np.float64).T
    assert (np.abs(y - exact) <= 8 * sd + np.abs(exact) * 2.0 ** -11 + 1e-6).all()
    net.backward()
    torch.cuda.synchronize()
    dy = host(b["fc.dy"]).reshape(4, -1)
    T = np.ascontiguousarray
    assert same(host(b["d:gap.y"]).reshape(4, -1), product(*quant_rows(dy), *quant_rows(T(w.T))))
    assert same(host(b["d:fc"]).reshape(1000, -1), product(*quant_rows(T(dy.T)), *quant_rows(T(x.T))))
    g = [host(t).copy() for t in muon["g"]]
    assert all(np.isfinite(v.astype(np.float32)).all() for v in g)
    bias0 = host(b["fc.bias"]).copy()
    net.update()
    torch.cuda.synchronize()
    for i in range(len(g)):
        check_update(w0[i], g[i], m0[i], host(muon["w"][i]), host(muon["m"][i]),
                     muon["descs"][i].scale, net.muon_lr, net.muon_momentum, net.wd, 1)
    wr, _ = oracle.sgd_f32(bias0, host(b["fc.dbias"]), np.zeros_like(bias0), net.lr, net.momentum,
                           net.wd)
    assert np.array_equal(host(b["fc.bias"]).view(np.uint16), wr.view(np.uint16))


def test_network_graph_replay_matches_eager():
    net = _net(optimizer="muon", classifier="int8")
    start = net.state()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        net.step()
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    net.load_state(start)
    eager = []
    for _ in range(3):
        net.step()
        torch.cuda.synchronize()
        eager.append(net.state())
    net.load_state(start)
    note("[gpu] capture of the step")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        net.step()
    net.load_state(start)
    for ref in eager:
        graph.replay()
        torch.cuda.synchronize()
        other = (torch.randn(1000, device="cuda") * 2).sum().item()  # eager work between
        assert np.isfinite(other)
        for a, b in zip(net.state(), ref):
            assert torch.equal(a.view(torch.int16), b.view(torch.int16))


class Layer:
    """A dense layer of a training program: buffers, workspaces and one step."""

    def __init__(self, t, i, o, seed):
        self.sizes = t, i, o
        self.x, self.w = gpu(acts(t, i, seed)), gpu(acts(o, i, seed + 1, 0.05))
        self.dy = gpu(acts(t, o, seed + 2, 1e-2))
        e = lambda *s: torch.empty(s, dtype=torch.float16, device="cuda")
        self.y, self.dx, self.dw, self.db = e(t, o), e(t, i), e(o, i), e(o)
        self.bias = gpu((0.1 * np.random.default_rng(seed).standard_normal(o)).astype(np.float16))
        self.m, self.mb = torch.zeros_like(self.w), torch.zeros_like(self.bias)
        self.wq, self.sw = F.int8_operand(o, i)
        self.wqt, self.swt = F.int8_operand(i, o)
        self.desc = F.int8_dense_desc(t, i, o)
        self.mats = F.muon_descs([(o, i, 1.5)])
        self.ws = F.workspace(F.fp16_int8_dense_workspace_bytes(self.desc))
        self.wsm = F.workspace(F.fp16_muon_workspace_bytes(self.mats, 3))

    def step(self):
        d = self.desc
        F.fp16_int8_dense_weights(d, self.w, self.wq, self.sw, self.wqt, self.swt, self.ws)
        F.fp16_int8_dense_fwd(d, self.x, self.wq, self.sw, self.bias, self.y, self.ws)
        F.fp16_int8_dense_bwd(d, self.x, self.dy, self.wqt, self.swt, self.dx, self.dw, self.db,
                              self.ws)
        F.fp16_muon_step(self.mats, [self.w], [self.dw], [self.m], 0.05, 0.9, 0.01, products=3,
                         ws=self.wsm)
        F.fp16_sgd_step(self.bias, self.db, self.mb, None, 0.05, 0.9, 0.0)

    def tensors(self):
        return [self.y, self.dx, self.dw, self.db, self.w, self.m, self.bias, self.mb]


def test_dense_layer_steps():
    require_gpu()
    L = Layer(70, 200, 136, 1)
    T = np.ascontiguousarray
    for k in range(4):
        x, w, dy, bias, m = (host(t).copy() for t in (L.x, L.w, L.dy, L.bias, L.m))
        note(f"[gpu] dense layer step {k}")
        L.step()
        torch.cuda.synchronize()
        assert same(host(L.y), product(*quant_rows(x), *quant_rows(w), bias))
        assert same(host(L.dx), product(*quant_rows(dy), *quant_rows(T(w.T))))
        dw = product(*quant_rows(T(dy.T)), *quant_rows(T(x.T)))
        assert same(host(L.dw), dw)
        check_update(w, dw, m, host(L.w), host(L.m), 1.5, 0.05, 0.9, 0.01, 3)
        # the next step's data
        L.x.copy_(torch.from_numpy(acts(70, 200, 50 + k)))
        L.dy.copy_(torch.from_numpy(acts(70, 136, 60 + k, 1e-2)))


def test_two_captured_programs_beside_each_other():
    """Each with its own workspaces, replayed on two streams at once, several times:
    the same bits as run alone."""
    require_gpu()
    shapes = [(70, 200, 136), (33, 512, 256)]
    ref = [Layer(*s, seed) for seed, s in enumerate(shapes)]
    for L in ref:
        for _ in range(4):
            L.step()
    torch.cuda.synchronize()
    both = [Layer(*s, seed) for seed, s in enumerate(shapes)]
    streams = [torch.cuda.Stream() for _ in both]
    graphs = []
    for L, s in zip(both, streams):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            L.step()  # the first step eagerly
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            L.step()
        graphs.append(g)
    for _ in range(3):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for L, R in zip(both, ref):
        for a, b in zip(L.tensors(), R.tensors()):
            assert torch.equal(a.view(torch.int16), b.view(torch.int16))
