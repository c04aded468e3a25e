"""ResNet-50's step with the classifier as a dense layer and dropout before it, and its
predictions, on the GPU: the new calls replayed on the inputs that the GPU's saw, graph
replays equal to eager steps, everything before the dropout as in the plain network."""

import numpy as np
import pytest
import torch

import head_oracle as O
from gpu_util import host, note, require_gpu
from paper_1911_07384_amd.network import ResNet50

pytestmark = pytest.mark.gpu


def make(**kw):
    require_gpu()
    net = ResNet50(n=4, image=64, seed=3, **kw)
    net.load_batch(3)
    return net


def flat(net, name, *shape):
    return host(net.buffers[name]).reshape(shape)


def test_step():
    note("[gpu] ResNet-50 step with a dense classifier and dropout")
    net, plain = make(classifier="dense", dropout=0.4), make()
    net.buffers["fc.bias"].copy_(torch.linspace(-1, 1, 1000).half())
    net.forward()
    plain.forward()
    torch.cuda.synchronize()
    assert torch.equal(net.buffers["gap.y"], plain.buffers["gap.y"])
    x0, x = flat(net, "gap.y", 4, -1), flat(net, "drop.y", 4, -1)
    assert np.array_equal(x, O.dropout(x0, None, 0.4, 3, 0, 0))
    w, bias = flat(net, "fc", 1000, -1), host(net.buffers["fc.bias"])
    net.backward()
    torch.cuda.synchronize()
    dy = flat(net, "fc.dy", 4, 1000)
    want = O.Dense(x, w, bias, dy=dy, z=None)
    O.close(flat(net, "fc.y", 4, 1000), want.y, want.y_err, "logits")
    O.close(flat(net, "d:fc", 1000, -1), want.dw, want.dw_err, "dW")
    dx = flat(net, "d:drop.y", 4, -1)
    O.close(dx, want.dx, want.dx_err, "d features")
    assert np.array_equal(flat(net, "d:gap.y", 4, -1), O.dropout(dx, None, 0.4, 3, 0, 0))
    # the bias' gradient: the exact sum of the stored gradient, rounded once
    db = torch.from_numpy(dy).double().sum(0)
    O.close(host(net.buffers["fc.dbias"]), db, O.HALF * db.abs() + O.TINY, "dbias")
    net.update()
    torch.cuda.synchronize()
    assert net.buffers["rng"].tolist() == [3, 1]
    net.forward()
    torch.cuda.synchronize()
    assert np.array_equal(flat(net, "drop.y", 4, -1),
                          O.dropout(flat(net, "gap.y", 4, -1), None, 0.4, 3, 1, 0))


@pytest.mark.parametrize("classifier", ["fp16", "int8", "dense"])
def test_graph_replay_matches_eager(classifier):
    net = make(classifier=classifier, dropout=0.25)
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
    assert not torch.equal(eager[0][0], eager[1][0])
    net.load_state(start)
    note(f"[gpu] capture of the step, classifier {classifier}")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        net.step()
    net.load_state(start)
    for ref in eager:
        graph.replay()
        torch.cuda.synchronize()
        assert np.isfinite((torch.randn(1000, device="cuda") * 2).sum().item())  # eager work
        for a, b in zip(net.state(), ref):
            assert torch.equal(a.view(torch.int16), b.view(torch.int16))


@pytest.mark.parametrize("classifier", ["fp16", "dense"])
def test_predictions(classifier):
    net = make(classifier=classifier, dropout=0.5)
    net.buffers["fc.bias"].copy_(torch.linspace(-1, 1, 1000).half())
    note("[gpu] predictions")
    out = net.predict(7)
    torch.cuda.synchronize()
    want = O.Dense(flat(net, "gap.y", 4, -1), flat(net, "fc", 1000, -1),
                   host(net.buffers["fc.bias"]))
    z = host(out["logits"])
    O.close(z, want.y, want.y_err, "logits")
    L = O.Logprob(z, 1.0, 7)
    assert np.array_equal(host(out["top_id"]), L.top_id)
    lab = net.buffers["labels"].cpu().long()
    assert (out["logp"].cpu().double() - L.lp.gather(1, lab[:, None])[:, 0]).abs().max() < 1e-5
    assert (out["stats"].cpu()[:, 2].double() - L.h).abs().max() < 1e-4
    # the labels made the predicted ones: accuracies
    net.buffers["labels"].copy_(out["top_id"][:, 0])
    net.buffers["labels"][0] = out["top_id"][0, 4]
    net.buffers["labels"][1] = out["top_id"][1, 5]
    e = net.evaluate()
    assert e["top1"] == 0.5 and e["top5"] == 0.75
    lab = net.buffers["labels"].cpu().long()
    assert abs(e["loss"] + L.lp.gather(1, lab[:, None]).mean().item()) < 1e-5
    assert abs(e["entropy"] - L.h.mean().item()) < 1e-4


def test_predictions_in_a_graph():
    net = make(classifier="dense")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        first = net.predict(5)
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    note("[gpu] capture of predictions")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = net.predict(5)
    for _ in range(3):
        for t in out.values():
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out[k], first[k]) for k in out)
