"""bench.with_update: the gradients that the update takes are scaled once to the norm that clipping allows.  On the host with the
calls written out in 64 bits, on the GPU with the library's."""
import math
from types import SimpleNamespace

import pytest
import torch

import bench
import paper_2503_01066_amd as package


class OnTheHost:
    """The calls of the package that with_update makes, in 64 bits."""
    embed_backward_workspace_bytes = staticmethod(package.embed_backward_workspace_bytes)
    grad_clip_workspace_bytes = staticmethod(package.grad_clip_workspace_bytes)

    @staticmethod
    def GradList(grads, outs=None):
        return list(zip(grads, [None] * len(grads) if outs is None else outs))

    @staticmethod
    def AdamwList(params, grads, m, v, masters=None, weight_decay=0.0):
        return list(zip(grads, m, v))

    @staticmethod
    def alch_embed_backward(ids, dX, vocab, dW_embed, workspace):
        dW_embed.copy_(torch.zeros(dW_embed.shape, dtype=torch.float64).index_add_(0, ids.long(), dX.double()))

    @staticmethod
    def alch_grad_clip(grads, max_norm, norm_out, workspace):
        norm = math.sqrt(sum(float(g.double().square().sum()) for g, _ in grads))
        norm_out.copy_(torch.tensor([norm, min(1.0, max_norm / norm)]))
        for g, o in grads:
            if o is not None:
                o.copy_(g.double() * norm_out[1].double())

    @staticmethod
    def alch_adamw_step(tensors, lr, grad_factor=None):
        for g, m, v in tensors:
            x = g.double() * (1.0 if grad_factor is None else float(grad_factor))
            m.copy_(0.9 * m.double() + 0.1 * x)
            v.copy_(0.999 * v.double() + 0.001 * x.square())


@pytest.mark.parametrize("device", ["cpu", pytest.param("cuda", marks=pytest.mark.gpu)])
@pytest.mark.parametrize("size", [1.0, 1e-3])  # the norm above max_norm and below
def test_moments_are_those_of_gradients_clipped_once(device, size):
    V, H, T = 40, 64, 32
    gen = torch.Generator().manual_seed(5)
    dt = torch.bfloat16
    rnd = lambda *s: (torch.randn(s, generator=gen) * size).to(dt).to(device)
    ids = torch.randint(0, V, (T,), generator=gen).to(torch.int32).to(device)
    W, emb, W_lm, gain = rnd(H, H), rnd(V, H), rnd(V, H), rnd(H)
    dW, dX = torch.empty_like(W), rnd(T, H)
    new = [rnd(H, H), rnd(H), rnd(V, H)]

    def backward(xf, rs, hooks, head):
        for to, value in zip([dW, *head], new):
            to.copy_(value)
        return dict(dX_embed=dX)

    base = OnTheHost if device == "cpu" else package
    lists = []

    class Calls:
        def __getattr__(self, name):
            return getattr(base, name)

        def AdamwList(self, params, grads, m, v, **kw):
            lists.append((grads, m, v))
            return base.AdamwList(params, grads, m, v, **kw)

    step = bench.with_update(SimpleNamespace(frozen_base=False), torch, Calls(), backward, [dict(Wq=W)], None, None, [dict(dWq=dW)], emb, ids, W_lm, gain)
    step(None, None)
    (grads, m, v), = lists
    table = torch.zeros((V, H), dtype=torch.float64, device=device).index_add_(0, ids.long(), dX.double()).to(dt)
    raw = [x.double() for x in new + [table]]
    norm = math.sqrt(sum(float(x.square().sum()) for x in raw))
    assert (norm > 1.0) == (size == 1.0)
    f = min(1.0, 1.0 / norm)
    # bf16: the table's gradient (of rounded sums in another order: a step) and a clipped gradient's rounding, 2^-8 each at most twice,
    # the rest is fp32; squares twice that
    for x, a, b in zip(raw, m, v):
        assert bool(((a.double() - 0.1 * f * x).abs() <= 4 * 2.0 ** -8 * 0.1 * f * x.abs() + 1e-30).all())
        assert bool(((b.double() - 0.001 * (f * x).square()).abs() <= 9 * 2.0 ** -8 * 0.001 * (f * x).square() + 1e-30).all())
