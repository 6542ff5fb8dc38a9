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


def test_hidden_sizes_beyond_32_bits_are_refused():
    """They would be cut to a small one, which has a workspace and rows of its own."""
    ids, wide = torch.zeros(3, dtype=torch.int32), torch.zeros(1, 1)
    for call in (lambda: A.alch_embed_forward(ids, wide.expand(4, 2 ** 32 + 8)), lambda: A.alch_embed_backward(ids, wide.expand(3, 2 ** 32 + 8), 4),
                 lambda: A.embed_backward_workspace_bytes(torch.float32, 4, 2 ** 32 + 8, 3),
                 lambda: A.embed_backward_workspace_bytes(torch.float32, 8 - 2 ** 32, 8, 3)):
        with pytest.raises(ValueError, match="32 bits"):
            call()


def test_steps_beyond_32_bits_are_refused(monkeypatch):
    z = lambda: torch.zeros(8)
    tensors, steps = A.AdamwList([z()], [z()], [z()], [z()]), []
    monkeypatch.setattr(B, "lib", lambda: SimpleNamespace(alch_adamw_step=lambda n, d, h, p, s: steps.append(p._obj.step) or 0))
    monkeypatch.setattr(B, "_place", lambda device, stream: tensors.made_on)
    for step in (2 ** 32 + 1, 2 ** 31, -2 ** 31 - 1):
        with pytest.raises(ValueError, match="32 bits"):
            A.alch_adamw_step(tensors, 1e-3, step=step)
    A.alch_adamw_step(tensors, 1e-3, step=2 ** 31 - 1)
    assert steps == [2 ** 31 - 1]


@pytest.mark.parametrize("hidden", [1, 8, 256, 487, 512, 513, 4096, 8192, 8200, 20000, 1 << 17, 1 << 20])
@pytest.mark.parametrize("vocab", [1, 1000, 1023, 128256, 2 ** 20])
def test_a_workspace_for_a_batch_serves_every_smaller_one(hidden, vocab):
    """A program sizes it once, for its largest batch: the size never falls with the number of tokens, over all lengths of parts and blocks."""
    tiles = -(-hidden // 512)
    at = {0, 1, 2, 511, 512, 513}
    for part in (8, 16, 32):  # parts of a length end where 4096 wavefronts have their own
        at |= {part * k + d for k in (4095 // tiles, 4096 // tiles, -(-4096 // tiles)) for d in (-1, 0, 1)}
    for blocks in (512,):     # blocks of the sort become longer
        at |= {blocks * size + d for size in (512, 768, 1024, 1280) for d in (-1, 0, 1)}
    at |= {1 << k for k in range(31)} | {(1 << k) - 24 for k in range(6, 31)} | {8176, 8192, 16000, 16352, 16384}
    at = sorted(n for n in at if n >= 0 and n * hidden <= 1 << 40)
    for dtype in (torch.bfloat16, torch.float32):
        sizes = [A.embed_backward_workspace_bytes(dtype, vocab, hidden, n) for n in at]
        falls = [(n, m) for n, m, a, b in zip(at, at[1:], sizes, sizes[1:]) if b < a]
        assert not falls and sizes[0] > 0
