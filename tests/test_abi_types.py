"""Element types that the binding refuses before a call reaches the library (CPU
tensors; nothing is launched)."""

import pytest
import torch

import paper_1911_07384_amd as F


class NoLibrary:
    """Whose entry points fail the test: they would run on host memory."""

    def __getattr__(self, name):
        return lambda *a: pytest.fail(f"{name} was called")


@pytest.fixture(autouse=True)
def no_library(monkeypatch):
    monkeypatch.setattr(F, "lib", NoLibrary)


def half(*s):
    return torch.zeros(s, dtype=torch.float16)


def test_binary16_entry_points_refuse_int8():
    """An int8 tensor holds half the bytes that its element count stands for there."""
    w, b = half(64), torch.zeros(64, dtype=torch.int8)
    conv = F.conv_desc(1, 8, 4, 4, 8, 1, 1)
    for args in ((b, w, w), (w, b, w), (w, w, b)):
        for sgd in (F.fp16_sgd_step, F.fp16_sgd_step_f16):
            with pytest.raises(TypeError):
                sgd(*args, None, 0.1, 0.9, 0.0, stream=0)
        with pytest.raises(TypeError):
            F.fp16_conv_fwd(conv, *args, stream=0)


T, I, O = 8, 16, 32  # noqa: E741
LAYER = dict(x=half(T, I), w=half(O, I), dy=half(T, O), y=half(T, O), dx=half(T, I), dw=half(O, I),
             bias=half(O), dbias=half(O))
for name, rows, cols in (("wq", O, I), ("wqt", I, O), ("q", T, I)):
    LAYER[name] = torch.zeros((rows, cols), dtype=torch.int8)
    LAYER["scale_" + name] = torch.zeros(rows)
DESC = F.int8_dense_desc(T, I, O)
WS = torch.zeros(1 << 16, dtype=torch.uint8)
CALLS = {
    "quant_rows": (("x", "q", "scale_q"), lambda x, q, s: F.fp16_int8_quant_rows(T, I, x, q, s, 0)),
    "quant_cols": (("x", "q", "scale_q"),
                   lambda x, q, s: F.fp16_int8_quant_cols(T, I, x, q, s, WS, None, 0)),
    "matmul": (("q", "scale_q", "wq", "scale_wq", "bias", "y"),
               lambda *a: F.fp16_int8_matmul(T, O, I, *a, stream=0)),
    "weights": (("w", "wq", "scale_wq", "wqt", "scale_wqt"),
                lambda *a: F.fp16_int8_dense_weights(DESC, *a, WS, stream=0)),
    "fwd": (("x", "wq", "scale_wq", "bias", "y"),
            lambda *a: F.fp16_int8_dense_fwd(DESC, *a, WS, stream=0)),
    "bwd": (("x", "dy", "wqt", "scale_wqt", "dx", "dw", "dbias"),
            lambda *a: F.fp16_int8_dense_bwd(DESC, *a, WS, stream=0)),
}


@pytest.mark.parametrize("call", CALLS)
def test_8_bit_layers_take_each_argument_in_its_type(call):
    names, f = CALLS[call]
    good = [LAYER[n] for n in names]
    with pytest.raises(pytest.fail.Exception):  # as it should be: the library's turn
        f(*good)
    for i, n in enumerate(names):
        for dtype in (torch.float16, torch.float32, torch.int8, torch.uint8, torch.bfloat16):
            if dtype != good[i].dtype:
                with pytest.raises(TypeError):
                    f(*good[:i], good[i].to(dtype), *good[i + 1:])
        if good[i].dim() == 2:
            with pytest.raises(ValueError):
                f(*good[:i], torch.zeros(good[i].shape[::-1], dtype=good[i].dtype).t(), *good[i + 1:])


def test_lists_of_matrices_fit_their_descriptors():
    """Each tensor of a list in binary16 and of its matrix's size at least, in every
    list and at every place of it."""
    shapes = [(8, 8), (16, 4), (5, 7)]
    d = F.muon_descs(shapes)
    good = [half(*s) for s in shapes]
    orth = lambda x, y: F.fp16_orthogonalize(d, x, y, ws=WS, stream=0)
    step = lambda w, g, m: F.fp16_muon_step(d, w, g, m, ws=WS, stream=0)
    for f, lists in ((orth, 2), (step, 3)):
        with pytest.raises(pytest.fail.Exception):
            f(*[good] * lists)
        with pytest.raises(pytest.fail.Exception):  # part of a larger buffer
            f(*[[half(100)] * 3] * lists)
        with pytest.raises(pytest.fail.Exception):  # addresses are the caller's matter
            f(*[[4096] * 3] * lists)
        for i in range(lists):
            for k in range(3):
                for bad, error in ((good[k].float(), TypeError), (good[k].to(torch.int8), TypeError),
                                   (good[k].flatten()[:-1], ValueError), (half(0), ValueError),
                                   (half(*shapes[k][::-1], 2)[:, :, 0].t(), ValueError)):
                    l = [list(good) for _ in range(lists)]
                    l[i][k] = bad
                    with pytest.raises(error):
                        f(*l)
