"""CPU-only checks around the lists of tensors and the counts and workspaces of the calls at the two ends of a training step."""
import ctypes as C
from types import SimpleNamespace

import pytest
import torch

import paper_2503_01066_amd as A
from paper_2503_01066_amd import binding as B


class Recorded:
    """Stands for a list's device array: notes the streams it is kept for."""

    def __init__(self):
        self.streams = []

    def record_stream(self, s):
        self.streams.append(s)


@pytest.mark.parametrize("call", ["clip", "adamw"])
def test_a_list_is_kept_for_the_stream_that_a_call_goes_to(monkeypatch, call):
    """Its memory belongs to the stream it was made on; a call on another one, be it given or the current one, has still to read it when the
    list is dropped."""
    t = lambda: torch.zeros(8)
    tensors = A.GradList([t()]) if call == "clip" else A.AdamwList([t()], [t()], [t()], [t()])
    library = SimpleNamespace(alch_grad_clip=lambda *a: 0, alch_adamw_step=lambda *a: 0)
    monkeypatch.setattr(B, "lib", lambda: library)
    tensors.dev, tensors.made_on = Recorded(), 7
    current = SimpleNamespace(cuda_stream=None)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: current)
    monkeypatch.setattr(B, "_place", lambda device, stream: current.cuda_stream if stream is None else stream.cuda_stream)

    def run(stream):
        if call == "clip":
            A.alch_grad_clip(tensors, 1.0, norm_out=torch.empty(2), workspace=torch.empty(16, dtype=torch.uint8), stream=stream)
        else:
            A.alch_adamw_step(tensors, 0.1, stream=stream)

    given = SimpleNamespace(cuda_stream=9)
    for at, stream, kept in ((7, None, []), (8, None, [current]), (7, given, [given]), (8, given, [given])):
        tensors.dev.streams, current.cuda_stream = [], at
        run(stream)
        assert tensors.dev.streams == kept, (at, stream)
