"""CPU-only checks of records and moments in 8 bits and of the policy loss: what the library and the binding refuse, before any GPU work."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2503_01066_amd as A
from paper_2503_01066_amd import binding as B

P = 1 << 40  # fake, aligned, never dereferenced: validation fails first
INVALID, SHAPE, WORKSPACE, UNSUPPORTED = -1, -2, -3, -5
FAR = 1 << 32


def _err():
    return A.lib().alch_last_error().decode()


def batch(lens=(3, 0, 5)):
    return A.Batch(np.concatenate([[0], np.cumsum(lens)]), device="cpu")


def entries(*over, n=1, rows=8):
    """Good streams, far apart, with what `over` says of each."""
    good = [dict(tensor=P + 8 * i * FAR, codes=P + (8 * i + 1) * FAR, scales=P + (8 * i + 2) * FAR, width=72, row_stride_bytes=144, dtype=1)
            for i in range(max(n, len(over)))]
    return (B.CQ8 * len(good))(*[B.CQ8(**dict(g, **(over[i] if i < len(over) else {}))) for i, g in enumerate(good)])


def test_structs_match_the_header():
    assert C.sizeof(B.CQ8) == 48 and C.sizeof(B.CPolicy) == 80 and C.sizeof(B.Adamw8Tensor) == 80
    assert A.lib().alch_policy_loss_workspace_bytes(5, 100) > 0


def test_pack_q8_refusals():
    L, b = A.lib(), batch()
    need = L.alch_capture_pack_workspace_bytes(8)

    def call(*over, b=b, mask=P + 99 * FAR, n=None, cap=8, idx=P + 100 * FAR, cu=P + 101 * FAR, st=P + 102 * FAR, ws=P + 103 * FAR, wsb=need, streams=True):
        e = entries(*over)
        return L.alch_capture_pack_q8(C.byref(b.c) if b else None, mask, len(e) if n is None else n, C.addressof(e) if streams else None, cap, idx, cu, st,
                                      ws, wsb, None)

    assert call(b=None) == INVALID and call(mask=None) == INVALID and call(mask=P + 1) == INVALID
    assert call(n=-1) == INVALID and call(streams=False) == INVALID and call(cap=-1) == INVALID
    for bad, status in ((dict(dtype=2), INVALID), (dict(width=0), SHAPE), (dict(width=-8), SHAPE), (dict(row_stride_bytes=143), SHAPE),
                        (dict(row_stride_bytes=142), SHAPE), (dict(dtype=0), SHAPE), (dict(tensor=None), INVALID), (dict(codes=None), INVALID),
                        (dict(scales=None), INVALID), (dict(tensor=P + 1), INVALID), (dict(codes=P + FAR + 8), INVALID), (dict(scales=P + 2 * FAR + 4), INVALID),
                        (dict(width=(1 << 31) + 1, row_stride_bytes=1 << 33), SHAPE), (dict(row_stride_bytes=1 << 41), SHAPE)):
        assert call({}, bad) == status and "stream 1" in _err(), bad
    assert call(idx=None) == INVALID and call(idx=P + 2) == INVALID and call(cu=None) == INVALID and call(st=None) == INVALID and call(st=P + 1) == INVALID
    assert call(wsb=need - 1) == WORKSPACE and call(ws=None) == WORKSPACE and call(ws=P + 2) == INVALID
    # memory that is written may not be memory of anything else of the call
    for bad in (dict(codes=P + 7 * 144 + 128), dict(scales=P), dict(codes=P + 2 * FAR), dict(scales=P + FAR + 560)):
        assert call(bad) == INVALID and "overlaps" in _err(), bad
    assert call({}, dict(codes=P + FAR)) == INVALID and "1: codes" in _err()
    assert call(idx=P) == INVALID and call(cu=P + FAR) == INVALID and call(st=P + 99 * FAR) == INVALID and call(ws=P + 100 * FAR) == INVALID
    assert call(idx=P + 101 * FAR) == INVALID and "overlaps" in _err()


def test_gather_q8_refusals():
    L, b = A.lib(), batch()

    def call(*over, n=None, cap=8, idx=P + 100 * FAR, st=P + 102 * FAR):
        e = entries(*over)
        return L.alch_capture_gather_q8(C.byref(b.c), len(e) if n is None else n, C.addressof(e), cap, idx, st, None)

    assert call(idx=None) == INVALID and "together" in _err() and call(st=None) == INVALID
    assert call(idx=None, st=None, cap=7) == SHAPE and "all of which" in _err()
    assert call(idx=P + 2) == INVALID and call(idx=P + FAR) == INVALID and "overlaps" in _err() and call(dict(width=0)) == SHAPE
    assert call(n=0) == 0 and call(cap=0) == 0  # nothing to do, nothing is launched


def test_expand_refusals():
    L = A.lib()

    def call(*over, n_rows=8, rows=P + 100 * FAR, held=9, n=None, tensors=True):
        e = entries(*over)
        return L.alch_record_expand(n_rows, rows, held, len(e) if n is None else n, C.addressof(e) if tensors else None, None)

    assert call(n_rows=-1) == INVALID and call(held=-1) == INVALID and call(n=-1) == INVALID and call(tensors=False) == INVALID
    assert call(n_rows=(1 << 31) + 1) == UNSUPPORTED and call(held=(1 << 31) + 1) == UNSUPPORTED
    assert call(rows=None, n_rows=10) == SHAPE and call(rows=P + 2) == INVALID
    for bad, status in ((dict(dtype=7), INVALID), (dict(width=0), SHAPE), (dict(row_stride_bytes=142), SHAPE), (dict(tensor=None), INVALID),
                        (dict(tensor=P + 1), INVALID), (dict(codes=P + FAR + 1), INVALID), (dict(scales=None), INVALID)):
        assert call({}, bad) == status and "tensor 1" in _err(), bad
    for bad in (dict(tensor=P + FAR), dict(tensor=P + 2 * FAR + 16), dict(tensor=P + 100 * FAR), dict(tensor=P + FAR + 9 * 72 - 8)):
        assert call(bad) == INVALID and "overlaps" in _err(), bad
    # column slices of one buffer are apart, others are not
    side = lambda at, **kw: dict(tensor=P + at, row_stride_bytes=288, **kw)
    assert call(side(0), side(144), n=2, n_rows=0) == 0
    assert call(side(0), side(142)) == INVALID and "0: dst overlaps 1: dst" in _err()
    assert call(side(144), side(0), side(288)) == INVALID  # (a column further than the row: the next row's first)
    assert call(side(0), dict(tensor=P + 144, row_stride_bytes=290)) == INVALID
    assert call(n_rows=0) == 0 and call(n=0, tensors=False) == 0 and call(n_rows=0, rows=None, held=0) == 0


def policy(**kw):
    good = dict(n_items=5, clip_low=0.2, clip_high=0.2, kl_coef=0.1, label=P, old_logp=P + FAR, advantage=P + 2 * FAR, weight=P + 3 * FAR, ref_logp=P + 4 * FAR,
                logp_out=P + 5 * FAR)
    return B.CPolicy(**dict(good, **kw))


def test_policy_loss_refusals():
    L = A.lib()
    need = L.alch_policy_loss_workspace_bytes(5, 100)

    def call(dt=1, V=100, x=P + 6 * FAR, ld=100, p=True, dx=P + 7 * FAR, ldg=100, loss=P + 8 * FAR, ws=P + 9 * FAR, wsb=need, **kw):
        pol = policy(**kw)
        return L.alch_policy_loss(dt, V, x, ld, C.byref(pol) if p else None, dx, ldg, loss, ws, wsb, None)

    assert call(dt=2) == INVALID and call(V=0) == SHAPE and call(V=(1 << 28) + 1) == UNSUPPORTED and call(p=False) == INVALID and call(n_items=-1) == INVALID
    nan, inf = float("nan"), float("inf")
    for bad in (dict(clip_low=-0.1), dict(clip_high=nan), dict(kl_coef=-1.0), dict(kl_coef=inf), dict(kl_coef=nan), dict(label=None), dict(label=P + 1),
                dict(old_logp=None), dict(advantage=P + 2 * FAR + 2), dict(weight=None), dict(ref_logp=None), dict(ref_logp=P + 3), dict(logp_out=P + 2)):
        assert call(**bad) == INVALID and "policy" in _err(), bad
    assert call(loss=None) == INVALID and call(loss=P + 2) == INVALID and call(wsb=need - 1) == WORKSPACE and call(ws=None) == WORKSPACE and call(ws=P + 8) == INVALID
    assert call(x=None) == INVALID and call(x=P + 8) == INVALID and call(dx=P + 8) == INVALID and call(ld=99) == SHAPE and call(ldg=99) == SHAPE
    assert call(ld=1 << 49) == UNSUPPORTED and call(ldg=1 << 60) == UNSUPPORTED
    assert call(dx=P + 6 * FAR, ldg=104) == SHAPE and "in place" in _err()
    assert call(dx=P + 6 * FAR + 16) == INVALID and "dlogits overlaps" in _err()
    assert call(dx=P + 6 * FAR + 16 * 62) == INVALID and call(logp_out=P) == INVALID and call(loss=P + 5 * FAR + 16) == INVALID and call(ws=P + 7 * FAR) == INVALID
    q = L.alch_policy_loss_workspace_bytes
    assert q(-1, 100) == 0 and q(5, 0) == 0 and q(5, (1 << 28) + 1) == 0 and q(0, 100) > 0
    sizes = [q(n, V) for V in (1000, 128256) for n in (0, 1, 2, 17, 100, 255, 256, 257, 1000, 100000, 1 << 30)]
    assert all(a <= b for a, b in zip(sizes[:11], sizes[1:11])) and all(a <= b for a, b in zip(sizes[11:], sizes[12:]))


def test_stack_backward_policy_refusals():
    L, b = A.lib(), batch()
    shape = A.make_shape(64, 4, 2, 16, 128, 1e-6, 1e4, "bf16")
    rows = np.array([0, 1, 1, 4, 7], np.int32)
    need = A.binding.stack_backward_workspace_bytes(shape, 0, 100, 8, 5)

    def call(shape=shape, rows=rows, p=True, loss=P + 8 * FAR, wsb=need, **kw):
        pol = policy(**dict(dict(item_row=P, item_row_host=rows.ctypes.data), **kw))
        return L.alch_stack_backward_policy(C.byref(shape), 0, 100, C.byref(b.c), None, None, None, P, P, P, C.byref(pol) if p else None, None, None, None,
                                            None, P, loss, None, P, wsb, None)

    assert call(p=False) == INVALID and "policy is NULL" in _err()
    assert call(n_items=9) == SHAPE and call(n_items=-1) == INVALID and call(item_row=None) == INVALID and call(item_row_host=None) == INVALID
    assert call(weight=None) == INVALID and call(kl_coef=-1.0) == INVALID and call(ref_logp=None) == INVALID and call(loss=None) == INVALID
    assert call(loss=P + 2) == INVALID and call(logp_out=P) == INVALID and "overlaps" in _err()
    assert call(rows=np.array([0, 1, 0, 4, 7], np.int32)) == SHAPE and "ascending" in _err()
    assert call(rows=np.array([0, 1, 2, 4, 8], np.int32)) == SHAPE and call(rows=np.array([-1, 1, 2, 4, 7], np.int32)) == SHAPE
    assert call(shape=A.make_shape(60, 4, 2, 16, 128, 1e-6, 1e4, "bf16")) == UNSUPPORTED
    assert call(wsb=need - 1) == WORKSPACE


def test_adamw8_refusals():
    L = A.lib()
    good = dict(param=P, grad=P, master=None, m=P, v=P, m_scale=P + 3, v_scale=P + 5, n=8, first=0, weight_decay=0.1, dtype=1)

    def call(n=None, dev=P + FAR, host=True, params=True, t=(), **kw):
        rows = [B.Adamw8Tensor(**dict(good, **r)) for r in (t or ({},))]
        h = (B.Adamw8Tensor * len(rows))(*rows)
        p = B.CAdamw(**dict(dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1), **kw))
        return L.alch_adamw8_step(len(rows) if n is None else n, dev, C.addressof(h) if host else None, C.byref(p) if params else None, 7, None)

    assert call(n=-1) == INVALID and call(n=4097) == UNSUPPORTED and call(dev=None) == INVALID and call(host=False) == INVALID and call(dev=P + 4) == INVALID
    assert call(params=False) == INVALID and call(step=0) == INVALID and call(beta1=1.0) == INVALID and call(beta2=-0.1) == INVALID and call(eps=-1.0) == INVALID
    assert call(schedule=P + 2) == INVALID and call(grad_factor=P + 1) == INVALID
    for k in ("param", "grad", "m", "v"):
        assert call(t=[{k: None}]) == INVALID and k in _err() and call(t=[{}, {k: P + 8}]) == INVALID and "tensor 1" in _err()
    assert call(t=[{"master": P + 4}]) == INVALID and call(t=[{"m_scale": None}]) == INVALID and call(t=[{"v_scale": None}]) == INVALID
    assert call(t=[{"n": -1}]) == SHAPE and call(t=[{"dtype": 7}]) == INVALID and call(t=[{"first": -1}]) == INVALID and call(t=[{"first": (1 << 62) + 1}]) == INVALID
    for k, a in (("m", 16), ("v", 16), ("m_scale", 1), ("v_scale", 1), ("param", 16)):
        assert call(t=[{k: P + FAR + 16, "n": 8}]) == INVALID and "overlaps" in _err(), k
        assert call(schedule=P + 5 * FAR, t=[{k: P + 5 * FAR}]) == INVALID and "schedule" in _err(), k
    assert call(t=[dict(n=0, param=None, grad=None, m=None, v=None, m_scale=None, v_scale=None)]) == 0 and call(n=0, dev=None, host=False) == 0


def test_lists_of_moments_in_8_bits():
    p = [torch.randn(5), torch.randn(0), torch.randn(3, 50).bfloat16()]
    state = lambda: [A.adamw8_state(x.shape, "cpu") for x in p]
    g = [torch.zeros_like(x) for x in p]
    m, v = state(), state()
    t = A.Adamw8List(p, g, m, v, masters=[None, None, torch.zeros(3, 50)], weight_decay=[0.1, 0, 0.2])
    rows = (B.Adamw8Tensor * 3).from_address(t.host_ptr)
    assert [(r.n, r.dtype, r.first) for r in rows] == [(5, 0, 0), (0, 0, 64), (150, 1, 64)]
    assert rows[2].m == m[2][0].data_ptr() and rows[2].v_scale == v[2][1].data_ptr() and m[2][1].numel() == 3
    assert bytes(t.dev.numpy()) == C.string_at(t.host_ptr, 240)
    assert [r.first for r in A.Adamw8List(p, g, state(), state(), first=[7, 1 << 40, 0]).host] == [7, 1 << 40, 0]
    with pytest.raises(ValueError, match="2 m for 3"):
        A.Adamw8List(p, g, state()[:2], state())
    with pytest.raises(ValueError, match="first"):
        A.Adamw8List(p, g, state(), state(), first=[0, 1, -2])
    with pytest.raises(ValueError, match=r"m\[0\]"):
        A.Adamw8List(p, g, [(c.int(), s) for c, s in state()], state())
    with pytest.raises(ValueError, match=r"v scales\[0\]"):
        A.Adamw8List(p, g, state(), [(c, s[:-1]) for c, s in state()])
    same = state()
    with pytest.raises(ValueError, match="overlaps"):
        A.Adamw8List(p, g, same, same)
    empty = A.Adamw8List([], [], [], [], device="cpu")
    assert empty.n == 0


def test_steps_and_seeds_beyond_32_bits_are_refused(monkeypatch):
    p, s = [torch.zeros(8)], lambda: [A.adamw8_state((8,), "cpu")]
    t = A.Adamw8List(p, [torch.zeros(8)], s(), s())
    monkeypatch.setattr(B, "_place", lambda device, stream: 0)
    for kw in (dict(step=1 << 31), dict(seed=1 << 32), dict(seed=-1)):
        with pytest.raises(ValueError, match="32 bits"):
            A.alch_adamw8_step(t, 0.1, **kw)


def test_items_of_a_policy_loss():
    f = lambda n=4: torch.zeros(n)
    label = torch.zeros(4, dtype=torch.int32)
    it = A.PolicyItems(label, f(), f(), f(), rows=[0, 1, 1, 2])
    assert it.rows.tolist() == [0, 1, 1, 2] and it.words[32:40] == bytes(8) and len(it.policy(0.2, 0.3, 0.1, f())) == C.sizeof(B.CPolicy)
    p = B.CPolicy.from_buffer_copy(it.policy(0.25, 0.5, 0.125, label))
    assert (p.n_items, p.clip_low, p.clip_high, p.kl_coef, p.label, p.ref_logp, p.item_row, p.logp_out) == (4, 0.25, 0.5, 0.125, label.data_ptr(), None, it.rows.data_ptr(), label.data_ptr())
    for bad in (dict(label=label.long()), dict(old=f(3)), dict(weight=f().double()), dict(ref_logp=f(8)[::2]), dict(rows=[0, 1])):
        a = dict(dict(label=label, old=f(), advantage=f(), weight=f(), ref_logp=None, rows=None), **bad)
        with pytest.raises(ValueError):
            A.PolicyItems(a["label"], a["old"], a["advantage"], a["weight"], ref_logp=a["ref_logp"], rows=a["rows"])
