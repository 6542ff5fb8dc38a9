"""Gradients that a backward call makes itself: with accumulate it adds to them, so that they begin as zeros; and what is asked of the
head's.  Without a GPU: the library is stood for by functions that look at what they are handed."""
import ctypes as C
from types import SimpleNamespace

import pytest
import torch

import paper_2503_01066_amd as A
from paper_2503_01066_amd import binding as B

H, V, T, F = 8, 6, 4, 16
SHAPE = A.make_shape(H, 2, 1, 4, F, 1e-5, 1e4, "f32")
BATCH = SimpleNamespace(c=B.CBatch(), total_tokens=T, max_seqlen=T)
WIDTHS = dict(Wq=(H, H), Wk=(4, H), Wv=(4, H), Wo=(H, H), Wg=(F, H), Wu=(F, H), Wd=(H, F), g1=(H,), g2=(H,))
CALLS = ("alch_layer_backward", "alch_layer_backward_lora", "alch_stack_backward", "alch_stack_backward_lora", "alch_stack_backward_dpo")


class Library:
    """The address of every gradient that a call was given."""

    def __getattr__(self, name):
        if name.endswith("workspace_bytes"):
            return lambda *a: 256
        return lambda *a: 0


@pytest.fixture
def library(monkeypatch):
    monkeypatch.setattr(B, "lib", lambda: Library())
    monkeypatch.setattr(B, "_stream_handle", lambda stream: 0)
    plain = torch.empty_like
    monkeypatch.setattr(torch, "empty_like", lambda t, **kw: plain(t, **kw).fill_(float("nan")))  # (whatever the memory held)


def run(name, **kw):
    W = {k: torch.ones(WIDTHS[k]) for k in A.WEIGHT_KEYS}
    record = {k: torch.ones(T, H) for k in A.RECORD_KEYS + ("LSE",)}
    lora = {"q": (torch.ones(2, H), torch.ones(H, 2))}
    X, gain, W_lm, labels = torch.ones(T, H), torch.ones(H), torch.ones(V, H), torch.zeros(T, dtype=torch.int32)
    if name == "alch_layer_backward":
        return A.alch_layer_backward(SHAPE, BATCH, record, W, X, **kw)
    if name == "alch_layer_backward_lora":
        return A.alch_layer_backward_lora(SHAPE, BATCH, record, W, lora, 2, 1.0, X, want=("Wq", "g1"), **kw)
    if name == "alch_stack_backward":
        return A.alch_stack_backward(SHAPE, BATCH, [record], [W], X, gain, W_lm, labels, **kw)
    if name == "alch_stack_backward_lora":
        return A.alch_stack_backward_lora(SHAPE, BATCH, [record], [W], [lora], 2, 1.0, X, gain, W_lm, labels, want=("Wq", "g1"), **kw)
    items = SimpleNamespace
    it = A.DpoItems([0, 1], [1, 2], [0, 1], torch.zeros(2), device="cpu")
    return A.alch_stack_backward_dpo(SHAPE, BATCH, [record], [W], X, gain, W_lm, it, None, None, None, 0.1, lora_layers=[lora], rank=2, **kw)


def gradients(out):
    found = {k: v for k, v in out.items() if k in ("dg_final", "dW_lm") and v is not None}
    for d in [out] + list(out.get("layers", [])):
        found.update({k: v for k, v in d.items() if k[:2] in ("dW", "dg", "dA", "dB") and v is not None})
    return found


@pytest.mark.parametrize("name", CALLS)
def test_gradients_that_are_added_to_begin_as_zeros(library, name):
    kw = dict(want_head=True) if name == "alch_stack_backward_lora" else {}
    made = gradients(run(name, accumulate=True, **kw))
    assert len(made) >= 4 and all(bool((g == 0).all()) for g in made.values()), {k: g.flatten()[0].item() for k, g in made.items()}
    written = gradients(run(name, **kw))
    assert written.keys() == made.keys()  # (nothing is cleared where all of it is written)
    assert all(bool(torch.isnan(g).all()) for g in written.values())


HEADS = [c for c in CALLS if "stack" in c]


@pytest.mark.parametrize("name", HEADS)
def test_head_gradients_that_are_given_and_not_wanted_are_refused(library, name):
    head = torch.zeros(H), torch.zeros(V, H)
    for given in (head, (None, head[1]), (head[0], None)):
        with pytest.raises(ValueError, match="head_grads"):
            run(name, head_grads=given, want_head=False)
    for kw in (dict(), dict(want_head=True)):  # (given tensors are wanted ones, whatever the call does without any)
        out = run(name, head_grads=head, **kw)
        assert out["dg_final"] is head[0] and out["dW_lm"] is head[1]
    assert run(name, head_grads=(None, head[1]))["dg_final"] is None
    out = run(name, want_head=False)
    assert out["dg_final"] is None and out["dW_lm"] is None
    assert run(name, head_grads=(None, None), want_head=False)["dW_lm"] is None
    without = run(name)
    assert (without["dW_lm"] is None) == (name == "alch_stack_backward_lora")


@pytest.mark.parametrize("given", [(torch.zeros(H),), (torch.zeros(H), torch.zeros(V, H), torch.zeros(1))])
def test_head_gradients_are_two(library, given):
    for name in HEADS:
        with pytest.raises(ValueError, match="head_grads: 2"):
            run(name, head_grads=given)
