"""ResNet-50's step with the classifier as a dense layer and dropout before it, planned on
the host (no kernels run)."""

import pytest
import torch

from paper_1911_07384_amd.network import ResNet50


def make(**kw):
    return ResNet50(n=1, image=64, device="cpu", **kw)


def test_options():
    for p in (-0.1, 1.5, float("nan")):
        with pytest.raises(ValueError):
            make(dropout=p)
    with pytest.raises(ValueError):
        make(classifier="linear")


def test_without_the_options_nothing_changes():
    net = make()
    kinds = {o.kind for o in net.fwd + net.bwd + net.upd}
    assert not kinds & {"dropout", "dropout_bwd", "rng_advance", "dense_fwd", "dense_bwd"}
    assert "rng" not in net.buffers and len(net.state()) == 4


@pytest.mark.parametrize("classifier", ["fp16", "int8", "dense"])
@pytest.mark.parametrize("dropout", [0.0, 0.3])
def test_program(classifier, dropout):
    net = make(classifier=classifier, dropout=dropout)
    fwd, bwd = [o.kind for o in net.fwd], [o.kind for o in net.bwd]
    want = {"fp16": ["conv_fwd"], "int8": ["int8_weights", "int8_fwd"], "dense": ["dense_fwd"]}
    at = fwd.index("avgpool_fwd")
    assert fwd[at:] == (["avgpool_fwd"] + (["dropout"] if dropout else []) + want[classifier]
                        + ["softmax_ce"])
    want = {"fp16": ["conv_dgrad", "conv_wgrad"], "int8": ["int8_bwd"], "dense": ["dense_bwd"]}
    n = len(want[classifier])
    assert bwd[:n] == want[classifier]
    assert bwd[n:n + 1 + bool(dropout)] == (["dropout_bwd"] if dropout else []) + ["avgpool_bwd"]
    assert ([o.kind for o in net.upd][-1] == "rng_advance") == bool(dropout)
    # every buffer a call reads is an input, a parameter or written earlier
    written = {"image", "labels", "fc.zero"} | {c["name"] for c in net.convs} | {"fc.bias"}
    for name, _ in net._bnspecs:
        written |= {name + ".gamma", name + ".beta"}
    grads = set()
    for op in net.prep + net.fwd + net.bwd:
        outs = [k for k in net._OUTPUTS[op.kind] if op.a.get(k) is not None]
        for k, v in op.a.items():
            if isinstance(v, str) and k not in outs and k not in ("mask_of", "conv"):
                assert v in net.buffers and v in written, (op.name, op.kind, v)
        written |= {op.a[k] for k in outs}
        if "dw" in op.a:
            grads.add(op.a["dw"])
    assert grads == {"d:" + c["name"] for c in net.convs}


def test_the_generators_state_is_kept():
    net = make(dropout=0.5, seed=9)
    st = net.state()
    assert st[-1].tolist() == [9, 0]
    net.buffers["rng"].add_(torch.tensor([0, 4]))
    net.load_state(st)
    assert net.buffers["rng"].tolist() == [9, 0]
