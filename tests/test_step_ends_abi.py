"""CPU-only checks of the entry points at the two ends of a training step (embedding rows and their gradient, clipping, the
weight update): what they refuse, before any GPU work, and the tables of tensors that two of them take."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2503_01066_amd as A
from paper_2503_01066_amd import binding as B

P = 0x10000  # fake, aligned, never dereferenced: validation fails first
INVALID, SHAPE, WORKSPACE, UNSUPPORTED = -1, -2, -3, -5


def _err():
    return A.lib().alch_last_error().decode()


def test_embed_forward_refusals():
    call = lambda dt=1, V=100, H=64, n=5, ids=P, W=P, X=2 * P: A.lib().alch_embed_forward(dt, V, H, n, ids, W, 1.0, X, None)
    assert call(dt=2) == INVALID and "dtype" in _err()
    assert call(V=0) == SHAPE and call(H=0) == SHAPE and call(H=-8) == SHAPE
    assert call(n=-1) == INVALID and call(n=(1 << 30) + 1) == UNSUPPORTED and call(H=(1 << 20) + 1) == UNSUPPORTED
    assert call(V=1 << 30, H=1 << 11) == UNSUPPORTED and "2^40" in _err()
    assert call(ids=None) == INVALID and "token_ids" in _err()
    assert call(ids=P + 2) == INVALID and "4-byte" in _err()
    assert call(W=None) == INVALID and call(W=P + 8) == INVALID and "W_embed" in _err()
    assert call(X=None) == INVALID and call(X=P + 2) == INVALID
    assert call(X=P) == INVALID and "overlaps" in _err()
    assert call(X=P + 99 * 128) == INVALID and call(X=P - 4 * 128) == INVALID
    assert call(n=0, ids=None, W=None, X=None) == 0  # nothing to do, nothing is launched


def test_embed_backward_refusals():
    L = A.lib()
    need = L.alch_embed_backward_workspace_bytes(1, 100, 64, 5)
    call = lambda dt=1, V=100, H=64, n=5, ids=P, dX=2 * P, dW=P, acc=0, ws=P, wsb=need: L.alch_embed_backward(
        dt, V, H, n, ids, dX, 1.0, dW, acc, ws, wsb, None)
    assert call(dt=-1) == INVALID and call(V=-1) == SHAPE and call(n=-1) == INVALID and call(n=(1 << 30) + 1) == UNSUPPORTED
    assert call(ids=None) == INVALID and call(ids=P + 1) == INVALID and call(dX=None) == INVALID and call(dX=P + 4) == INVALID
    assert call(dW=None) == INVALID and call(dW=P + 8) == INVALID and "dW_embed" in _err()
    assert call(dX=P + 99 * 128) == INVALID and "overlaps" in _err() and call(dX=P - 4 * 128) == INVALID
    assert call(wsb=need - 1) == WORKSPACE and call(ws=None) == WORKSPACE and call(ws=P + 8) == INVALID
    assert call(n=0, acc=1, ids=None, dX=None, dW=None, ws=None) == 0
    q = L.alch_embed_backward_workspace_bytes
    assert q(1, 100, 64, 0) > 0 and q(0, 0, 64, 5) == 0 and q(3, 100, 64, 5) == 0 and q(1, 100, 64, -1) == 0
    assert q(1, 128256, 4096, 16384) >= 128256 * 4 + 16384 * 8
    assert q(1, 1 << 20, 1 << 20, 1 << 20) > 1 << 38 and q(1, 2 ** 31 - 1, 512, 1 << 30) > 1 << 36  # (the largest: no overflow on the way)
    assert q(1, (1 << 20) + 1, 1 << 20, 5) == 0 and q(1, 5, 1 << 20, (1 << 20) + 1) == 0


def _grads(*rows):
    return (B.GradTensor * max(len(rows), 1))(*[B.GradTensor(*r) for r in rows])


def test_grad_clip_refusals():
    L = A.lib()
    need = L.alch_grad_clip_workspace_bytes()
    good = (P, 2 * P, 64, 1, 0)

    def call(rows=(good,), n=None, dev=P, host=True, max_norm=1.0, out=P, ws=P, wsb=need):
        h = _grads(*rows)
        return L.alch_grad_clip(len(rows) if n is None else n, dev, C.addressof(h) if host else None, max_norm, out, ws, wsb, None)

    assert call(n=-1) == INVALID and call(n=4097) == UNSUPPORTED and "4096" in _err()
    assert call(dev=None) == INVALID and call(host=False) == INVALID and call(dev=P + 4) == INVALID
    assert call([(P, None, -1, 1, 0)]) == SHAPE and call([(P, None, 8, 2, 0)]) == INVALID
    assert call([(None, None, 8, 1, 0)]) == INVALID and "grad is NULL" in _err()
    assert call([(P + 2, None, 8, 1, 0)]) == INVALID and call([(P, P + 8, 8, 1, 0)]) == INVALID
    assert call([good, (P, P + 64, 64, 1, 0)]) == INVALID and "tensor 1: out overlaps" in _err()
    assert call([(P, P - 64, 64, 1, 0)]) == INVALID
    assert call([(P, None, 1 << 40, 1, 0), (P, None, 1, 1, 0)]) == UNSUPPORTED and "2^40" in _err()
    assert call([(P, None, (1 << 62) + 5, 1, 0)] * 4) == UNSUPPORTED
    assert call(max_norm=-1.0) == INVALID and call(max_norm=float("nan")) == INVALID
    assert call(out=None) == INVALID and call(out=P + 2) == INVALID
    assert call(wsb=need - 1) == WORKSPACE and call(ws=None) == WORKSPACE and call(ws=P + 8) == INVALID


def test_adamw_refusals():
    L = A.lib()
    good = dict(param=P, grad=P, master=None, m=P, v=P, n=8, weight_decay=0.1, dtype=1)

    def call(n=None, dev=P, host=True, params=True, t=(), **kw):
        rows = [B.AdamwTensor(**dict(good, **r)) for r in (t or ({},))]
        h = (B.AdamwTensor * len(rows))(*rows)
        p = B.CAdamw(**dict(dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1), **kw))
        return L.alch_adamw_step(len(rows) if n is None else n, dev, C.addressof(h) if host else None, C.byref(p) if params else None, None)

    assert call(n=-1) == INVALID and call(n=4097) == UNSUPPORTED and call(dev=None) == INVALID and call(host=False) == INVALID
    assert call(params=False) == INVALID and "params" in _err()
    assert call(step=0) == INVALID and "step" in _err() and call(step=-3) == INVALID
    for bad in (1.0, -0.1, float("nan")):
        assert call(beta1=bad) == INVALID and call(beta2=bad) == INVALID
    assert call(eps=-1e-8) == INVALID and call(eps=float("nan")) == INVALID
    assert call(schedule=P + 2) == INVALID and call(grad_factor=P + 1) == INVALID
    for k in ("param", "grad", "m", "v"):
        assert call(t=[{k: None}]) == INVALID and k in _err()
        assert call(t=[{}, {k: P + 8}]) == INVALID and "tensor 1" in _err()
    assert call(t=[{"master": P + 4}]) == INVALID and call(t=[{"n": -1}]) == SHAPE and call(t=[{"dtype": 7}]) == INVALID
    assert call(t=[{"n": 0, "param": None, "grad": None, "m": None, "v": None}]) == 0  # nothing to do
    assert call(n=0, dev=None, host=False) == 0


def test_structs_match_the_header():
    assert C.sizeof(B.GradTensor) == 32 and C.sizeof(B.AdamwTensor) == 56 and C.sizeof(B.CAdamw) == 56


def test_tables_hold_what_the_library_reads():
    g = [torch.randn(5), torch.randn(0), torch.randn(3, 4).bfloat16()]
    out = [None, None, torch.empty(3, 4, dtype=torch.bfloat16)]
    t = A.GradList(g, out)
    rows = (B.GradTensor * 3).from_address(t.host_ptr)
    assert [(r.n, r.dtype) for r in rows] == [(5, 0), (0, 0), (12, 1)]
    assert [r.grad or 0 for r in rows] == [x.data_ptr() for x in g] and [r.out or 0 for r in rows] == [0, 0, out[2].data_ptr()]
    assert bytes(t.dev.numpy()) == C.string_at(t.host_ptr, 96)
    p = [torch.randn(4).bfloat16(), torch.randn(2)]
    f = lambda: [torch.zeros(4), torch.zeros(2)]
    m, v, w = f(), f(), [torch.zeros(4), None]
    t = A.AdamwList(p, [x.clone() for x in p], m, v, masters=w, weight_decay=[0.1, 0.0])
    rows = (B.AdamwTensor * 2).from_address(t.host_ptr)
    assert [r.param for r in rows] == [x.data_ptr() for x in p] and [r.m for r in rows] == [x.data_ptr() for x in m]
    assert [r.v for r in rows] == [x.data_ptr() for x in v] and (rows[0].master, rows[1].master) == (w[0].data_ptr(), None)
    assert [(r.n, r.dtype) for r in rows] == [(4, 1), (2, 0)] and rows[0].weight_decay == np.float32(0.1) and rows[1].weight_decay == 0


def test_tables_refuse_what_would_race_or_be_misread():
    a = torch.zeros(64)
    with pytest.raises(ValueError, match="outs.1. overlaps"):
        A.GradList([torch.zeros(8), torch.zeros(8)], [a[:8], a[4:12]])
    with pytest.raises(ValueError, match="overlaps"):
        A.GradList([a[:8], a[8:16]], [a[8:16], None])          # the output of one is the input of another
    with pytest.raises(ValueError, match="overlaps"):
        A.GradList([a[:8], a[:8]], [a[:8], a[:8]])             # one gradient twice, in place
    A.GradList([a[:8], a[:8], a])                              # (only read: legal)
    A.GradList([a[:8], a[8:16]], [a[:8], a[8:16]])             # in place, side by side
    with pytest.raises(ValueError, match="contiguous"):
        A.GradList([torch.zeros(4, 4).t()])
    with pytest.raises(ValueError, match="shape"):
        A.GradList([torch.zeros(4)], [torch.zeros(5)])
    with pytest.raises(TypeError, match="float16"):
        A.GradList([torch.zeros(4).half()])
    with pytest.raises(ValueError, match="2 outs for 1"):
        A.GradList([torch.zeros(4)], [None, None])
    z = lambda: torch.zeros(8)
    p = z()
    with pytest.raises(ValueError, match="overlaps"):
        A.AdamwList([p, p], [z(), z()], [z(), z()], [z(), z()])  # tied weights twice
    with pytest.raises(ValueError, match="overlaps"):
        A.AdamwList([p], [p], [z()], [z()])
    g = z()
    with pytest.raises(ValueError, match="overlaps"):
        A.AdamwList([p], [g], [z()], [g])
    A.AdamwList([z(), z()], [g, g], [z(), z()], [z(), z()])     # one gradient for two weights: only read
    with pytest.raises(ValueError, match=r"v\[0\]"):
        A.AdamwList([z().bfloat16()], [z().bfloat16()], [z()], [z().bfloat16()])
    with pytest.raises(ValueError, match="weight_decay"):
        A.AdamwList([z()], [z()], [z()], [z()], weight_decay=[0.1, 0.1])


def test_calls_refuse_tensors_that_are_not_on_the_current_device():
    ids, W = torch.zeros(3, dtype=torch.int32), torch.zeros(5, 8)
    for call in (lambda: A.alch_embed_forward(ids, W), lambda: A.alch_embed_backward(ids, torch.zeros(3, 8), 5),
                 lambda: A.alch_grad_clip(A.GradList([W]), 1.0),
                 lambda: A.alch_adamw_step(A.AdamwList([W], [W.clone()], [W.clone()], [W.clone()]), 1e-3)):
        with pytest.raises(ValueError, match="cpu"):
            call()


def test_counts_beyond_32_bits_are_refused():
    """The library takes 32 bits: a count that a conversion would cut to a small one is refused in front of it."""
    import torch
    ids, many = torch.zeros(3, dtype=torch.int32), torch.zeros(1, dtype=torch.int32).expand(2 ** 32 + 3)
    for call in (lambda: A.alch_embed_forward(many, torch.zeros(4, 8)), lambda: A.alch_embed_backward(ids, torch.zeros(3, 8), 2 ** 32 + 4),
                 lambda: A.alch_embed_backward(many, torch.zeros(1, 1).expand(2 ** 32 + 3, 1), 4),
                 lambda: A.embed_backward_workspace_bytes(torch.float32, 2 ** 32 + 4, 8, 3), lambda: A.embed_backward_workspace_bytes(torch.float32, 4, 8, 2 ** 31)):
        with pytest.raises(ValueError, match="more than 2.31 - 1"):
            call()


def test_scratch_and_ids_that_outputs_share_are_refused():
    """Sorted tokens that something else writes over would be followed to wherever they point."""
    L, far = A.lib(), 1 << 40
    need = L.alch_embed_backward_workspace_bytes(1, 100, 64, 5)
    call = lambda ids=far, dX=2 * far, dW=3 * far, ws=4 * far, acc=0: L.alch_embed_backward(1, 100, 64, 5, ids, dX, 1.0, dW, acc, ws, need, None)
    for acc in (0, 1):
        assert call(ws=3 * far + 99 * 128, acc=acc) == INVALID and "workspace overlaps dW_embed" in _err()
        assert call(ws=2 * far + 4 * 128, acc=acc) == INVALID and "workspace overlaps dX" in _err()
        assert call(ids=4 * far + need - 4, acc=acc) == INVALID and "workspace overlaps token_ids" in _err()
        assert call(ids=3 * far - 16, acc=acc) == INVALID and "dW_embed overlaps token_ids" in _err()
    assert L.alch_embed_backward(1, 100, 64, 0, None, None, 1.0, far, 0, far, need, None) == INVALID and "workspace overlaps dW_embed" in _err()
    assert L.alch_embed_forward(1, 100, 64, 5, far + 4 * 128 + 124, 2 * far, 1.0, far, None) == INVALID and "X overlaps token_ids" in _err()
    rows, size = _grads((far, None, 64, 1, 0)), L.alch_grad_clip_workspace_bytes()
    assert L.alch_grad_clip(1, P, C.addressof(rows), 1.0, 2 * far + size - 4, 2 * far, size, None) == INVALID and "workspace overlaps norm_out" in _err()
