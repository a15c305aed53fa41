"""restore_weight_f8 on a stream that is not the caller's current one: its scratch is kept from reuse until that stream has passed the call (no GPU: the
streams and the calls are stand-ins)."""
import contextlib

import pytest
import torch

import paper_2410_23918_amd as B


class Scratch:
    device = "cuda:0"

    def __init__(self):
        self.recorded = []

    def record_stream(self, stream):
        self.recorded.append(stream)


@pytest.mark.parametrize("stream,kept", [("side", ["side"]), ("main", []), (None, [])])
def test_scratch_of_the_caller(monkeypatch, stream, kept):
    current = ["main"]

    @contextlib.contextmanager
    def entered(s):
        current.append(s)
        yield
        current.pop()

    B.quantise_weight_f8   # loads f8.py
    from paper_2410_23918_amd import f8
    monkeypatch.setattr(torch.cuda, "stream", entered)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: current[-1])
    monkeypatch.setattr(f8, "quantise_weight_f8", lambda w, out=None, stream=None: (w, stream))
    monkeypatch.setattr(B.PackedStack, "restore_weight", lambda self, n_loaded, w_dense=None, stream=None: w_dense)
    scratch = Scratch()
    assert B.PackedStack.restore_weight_f8(object.__new__(B.PackedStack), 3, w_dense=scratch, stream=stream) == (scratch, stream)
    assert scratch.recorded == kept
