"""The dense head's binding takes no workspace for larger than it is; nothing is launched."""

import pytest
import torch

import paper_1911_07384_amd as F

A, B, C, D, E = (0x1000000000 * k for k in range(1, 6))  # far apart, aligned


def calls(ws, ws_bytes):
    d, lp = F.dense_desc(24, 40, 56, "gelu"), F.logprob_desc(1, 1 << 20, top=64)
    kw = dict(ws=ws, ws_bytes=ws_bytes, stream=0)
    return [lambda: F.fp16_dense_fwd(F.dense_desc(40, 41, 56), A, B, None, None, C, **kw),
            lambda: F.fp16_dense_bwd(d, A, B, C, D, E, None, **kw),
            lambda: F.fp16_logprobs(lp, A, None, None, B, C, D, **kw)]


@pytest.fixture
def no_launch(monkeypatch):
    """A call that passes the binding's checks says so in place of being made."""
    class Reached(Exception):
        pass

    class Lib:
        def __getattr__(self, name):
            def call(*a):
                raise Reached(name)
            return call
    monkeypatch.setattr(F, "_device", lambda: -1)
    monkeypatch.setattr(F, "lib", Lib)
    return Reached


def test_bytes_past_the_tensor(no_launch):
    ws = torch.zeros(64, dtype=torch.uint8)
    for n in (65, 1 << 30, -1):
        for call in calls(ws, n):
            with pytest.raises(ValueError, match="ws has 64 bytes"):
                call()
    for n in (None, 0, 64):
        for call in calls(ws, n):
            with pytest.raises(no_launch):
                call()


def test_negative_bytes_of_an_address(no_launch):
    for call in calls(1 << 40, -1):
        with pytest.raises(ValueError, match="ws_bytes"):
            call()
    for call in calls(1 << 40, 1 << 30):
        with pytest.raises(no_launch):
            call()


def test_a_workspace_that_is_too_small_is_refused(monkeypatch):
    monkeypatch.setattr(F, "_device", lambda: -1)
    for call in calls(torch.zeros(64, dtype=torch.uint8), 64):
        with pytest.raises(F.Fp16Error, match="WORKSPACE"):
            call()
