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


FAR = 1 << 40  # (addresses that are compared, never followed)
INVALID = -1


def _err():
    return A.lib().alch_last_error().decode()


def test_clipping_refuses_scratch_and_results_inside_its_gradients():
    """Work-groups read the sums for themselves while others store clipped values already."""
    L = A.lib()
    need = L.alch_grad_clip_workspace_bytes()

    def call(norm_out=3 * FAR, ws=4 * FAR, rows=((FAR, None, 0, 1, 0), (FAR, 2 * FAR, 1000, 1, 0), (FAR + 4096, None, 1000, 0, 0)), dev=64):
        h = (B.GradTensor * len(rows))(*[B.GradTensor(*r) for r in rows])
        return L.alch_grad_clip(len(rows), dev, C.addressof(h), 1.0, norm_out, ws, need, None)

    for at in (2 * FAR, 2 * FAR + 1984, 2 * FAR - need + 16):
        assert call(ws=at) == INVALID and "tensor 1: workspace overlaps out" in _err()
    assert call(ws=FAR + 1984) == INVALID and "tensor 1: workspace overlaps grad" in _err()
    assert call(ws=FAR + 4096 + 3984) == INVALID and "tensor 2: workspace overlaps grad" in _err()
    assert call(norm_out=2 * FAR + 1996) == INVALID and "tensor 1: norm_out overlaps out" in _err()
    assert call(norm_out=FAR - 4) == INVALID and "tensor 1: norm_out overlaps grad" in _err()
    assert call(norm_out=FAR + 8092) == INVALID and "tensor 2: norm_out overlaps grad" in _err()
    # the table, which all work-groups read
    assert call(dev=4 * FAR + need - 8) == INVALID and "workspace overlaps tensors" in _err()
    assert call(dev=3 * FAR - 88) == INVALID and "norm_out overlaps tensors" in _err()
    assert call(dev=2 * FAR + 1992) == INVALID and "tensor 1: tensors overlaps out" in _err()


def test_the_update_refuses_a_factor_or_schedule_inside_what_it_writes():
    L = A.lib()
    good = dict(param=FAR, grad=2 * FAR, master=3 * FAR, m=4 * FAR, v=5 * FAR, n=1000, weight_decay=0.0, dtype=1)

    def call(dev=64, **kw):
        rows = [B.AdamwTensor(**dict(good, n=0)), B.AdamwTensor(**good)]
        h = (B.AdamwTensor * 2)(*rows)
        p = B.CAdamw(**dict(dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1), **kw))
        return L.alch_adamw_step(2, dev, C.addressof(h), C.byref(p), None)

    for name, at, size in (("param", FAR, 2000), ("master", 3 * FAR, 4000), ("m", 4 * FAR, 4000), ("v", 5 * FAR, 4000)):
        for inside in (at, at + size - 4):
            assert call(grad_factor=inside) == INVALID and "tensor 1: grad_factor overlaps %s" % name in _err()
            assert call(schedule=inside) == INVALID and "tensor 1: schedule overlaps %s" % name in _err()
        assert call(dev=at - 104) == INVALID and "tensor 1: tensors overlaps %s" % name in _err()
        assert call(schedule=at - 4) == INVALID and "tensor 1: schedule overlaps %s" % name in _err()
