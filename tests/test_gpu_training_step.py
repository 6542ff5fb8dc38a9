"""A whole training step through the public entry points, as a program with a table shared by embedding and head runs it: embedding
rows, layers, cross-entropy and backward walk, the table's second gradient added to the head's, clipping over all gradients, the
update of all weights.  Gradients against the oracle in 64 bits and against differences of its loss; captured and replayed."""
import ctypes

import numpy as np
import pytest
import torch

import synth_inputs as synth
from helpers import TOL, TORCH_DT, to_dev, to_np, f64, rel_err, oracle_shape, alch_shape
from oracle import stack_backward_recompute, WEIGHT_KEYS
from oracle.stack import stack_loss

pytestmark = pytest.mark.gpu
SCALE, MAX_NORM, HYPER = 4.0, 0.05, dict(lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-6, step=5)


class Step:
    def __init__(self, shape_name, dtype, lens, V, L, wstd):
        import paper_2503_01066_amd as A
        self.A, self.dtype, self.L, self.V, self.cu = A, dtype, L, V, synth.ragged_cu(lens)
        shp, T = synth.shape_dict(shape_name), int(self.cu[-1])
        self.shp, self.shape, self.batch = shp, alch_shape(shp, dtype), A.Batch(self.cu)
        r = np.random.default_rng(3)
        self.ids = r.integers(0, V, T).astype(np.int32)
        self.ids[::7] = 11                        # an id that occurs often
        self.labels = np.full(T, -1, np.int32)
        for a, b in zip(self.cu[:-1], self.cu[1:]):
            self.labels[a:b - 1] = self.ids[a + 1:b]
        self.host = [synth.layer_weights(shp, 10 * l, dtype, std=wstd, gain_std=0.1) for l in range(L)]
        self.table = synth.normal(r, (V, shp["hidden"]), wstd, dtype)
        self.gain = synth.quantize(1.0 + 0.1 * r.standard_normal(shp["hidden"]).astype(np.float32), dtype)
        dev = lambda a: to_dev(a, dtype)
        self.W, self.E, self.g = [{k: dev(v) for k, v in W.items()} for W in self.host], dev(self.table), dev(self.gain)
        self.dev_ids, self.dev_labels = torch.from_numpy(self.ids).cuda(), torch.from_numpy(self.labels).cuda()
        H = shp["hidden"]
        empty = lambda *s: torch.empty(s, dtype=TORCH_DT[dtype], device="cuda")
        self.acts = [empty(T, H) for _ in range(L + 1)]
        QD, KD, F = shp["n_q_heads"] * shp["head_dim"], shp["n_kv_heads"] * shp["head_dim"], shp["ffn"]
        self.recs = [dict({k: empty(T, w) for k, w in dict(X2=H, Q=QD, K=KD, V=KD, O=QD, G=F, U=F).items()}, X=self.acts[l],
                          LSE=torch.empty((T, shp["n_q_heads"]), device="cuda")) for l in range(L)]
        self.grads = [{"d" + k: torch.empty_like(v) for k, v in W.items()} for W in self.W]
        ws = lambda n: torch.empty(n, dtype=torch.uint8, device="cuda")
        longest = max(lens)
        self.ws = [ws(A.lib().alch_layer_forward_workspace_bytes(ctypes.byref(self.shape), T, longest)),
                   ws(A.stack_backward_workspace_bytes(self.shape, L, V, T, longest)),
                   ws(A.embed_backward_workspace_bytes(TORCH_DT[dtype], V, H, T)), ws(A.grad_clip_workspace_bytes())]
        self.params = [W[k] for W in self.W for k in WEIGHT_KEYS] + [self.g, self.E]
        self.start = [p.clone() for p in self.params]
        self.masters = [p.float() for p in self.params] if dtype == "bf16" else None
        self.m, self.v = [torch.zeros(p.shape, device="cuda") for p in self.params], [torch.full(p.shape, 1e-6, device="cuda") for p in self.params]
        self.norm = torch.empty(2, device="cuda")
        self.head_grads = (torch.empty_like(self.g), torch.empty_like(self.E))
        g = [self.grads[l]["d" + k] for l in range(L) for k in WEIGHT_KEYS] + list(self.head_grads)
        self.all_grads, self.clip = g, A.GradList(g, g)
        self.adamw = A.AdamwList(self.params, g, self.m, self.v, masters=self.masters, weight_decay=[0.0 if p.dim() == 1 else 0.1 for p in self.params])

    def gradients(self):
        A = self.A
        A.alch_embed_forward(self.dev_ids, self.E, scale=SCALE, X=self.acts[0])
        for l in range(self.L):
            A.alch_layer_forward(self.shape, self.batch, self.acts[l], self.W[l], workspace=self.ws[0], rec=self.recs[l], Y=self.acts[l + 1])
        out = A.alch_stack_backward(self.shape, self.batch, self.recs, self.W, self.acts[-1], self.g, self.E, self.dev_labels,
                                    grads_layers=self.grads, workspace=self.ws[1], head_grads=self.head_grads)
        A.alch_embed_backward(self.dev_ids, out["dX_embed"], self.V, scale=SCALE, dW_embed=out["dW_lm"], accumulate=True, workspace=self.ws[2])
        return out

    def update(self):
        self.A.alch_grad_clip(self.clip, MAX_NORM, norm_out=self.norm, workspace=self.ws[3])
        self.A.alch_adamw_step(self.adamw, **HYPER)

    def reset(self):
        for p, s in zip(self.params, self.start):
            p.copy_(s)
        for i in range(len(self.params)):
            self.m[i].zero_()
            self.v[i].fill_(1e-6)
            if self.masters:
                self.masters[i].copy_(self.start[i])

    def state(self):
        torch.cuda.synchronize()
        return [x.clone() for x in self.params + self.m + self.v + (self.masters or []) + [self.norm]]


@pytest.mark.parametrize("dtype,shape_name,lens,V,wstd", [("f32", "tiny", [5, 1, 0, 8], 53, 0.3), ("bf16", "medium", [200, 150], 1024, 0.05)])
def test_step_against_oracle_and_differences(dtype, shape_name, lens, V, wstd):
    s = Step(shape_name, dtype, lens, V, 2, wstd)
    out = s.gradients()
    g = s.all_grads
    assert out["dg_final"].data_ptr() == g[-2].data_ptr() and out["dW_lm"].data_ptr() == g[-1].data_ptr()
    raw = [x.clone() for x in g]
    s.update()
    torch.cuda.synchronize()

    osh, Ws, E, gain = oracle_shape(s.shp), [f64(W) for W in s.host], s.table.astype(np.float64), s.gain.astype(np.float64)
    X0 = SCALE * E[s.ids]
    ref = stack_backward_recompute(osh, s.cu, None, X0, Ws, gain, E, s.labels)
    np.add.at(ref["dW_lm"], s.ids, SCALE * ref["dX_embed"])
    want = [ref["layers"][l]["d" + k] for l in range(2) for k in WEIGHT_KEYS] + [ref["dg_final"], ref["dW_lm"]]
    for i, (a, b) in enumerate(zip(raw, want)):
        assert rel_err(to_np(a), b) <= TOL[dtype], i
    # the norm of gradients that are each within that bar of the oracle's
    total = np.sqrt(sum(float((b ** 2).sum()) for b in want))
    slack = np.sqrt(sum(b.size * (TOL[dtype] * np.abs(b).max()) ** 2 for b in want))
    norm, factor = s.norm.tolist()
    assert abs(norm - total) <= slack + 2.0 ** -23 * total and norm > MAX_NORM
    # clipped in place, and every weight moved by the clipped gradient it was handed
    u, half = 2.0 ** -24, torch.finfo(TORCH_DT[dtype]).eps / 2
    for i, (p, p0, clipped, r) in enumerate(zip(s.params, s.start, g, raw)):
        c = r.double() * factor
        assert bool(((clipped.double() - c).abs() <= (2 * u + half) * c.abs() + 1e-44).all()), i
        m, v = 0.1 * clipped.double(), 0.95 * 1e-6 + 0.05 * clipped.double() ** 2
        change = m / (1 - 0.9 ** 5) / ((v / (1 - 0.95 ** 5)).sqrt() + 1e-6) + (0.0 if p.dim() == 1 else 0.1) * p0.double()
        w = p0.double() - 1e-3 * change
        assert bool(((p.double() - w).abs() <= (u + half) * w.abs() + 1e-3 * 32 * u * (change.abs() + p0.double().abs())).all()), i

    # the table's whole gradient against differences of the oracle's loss, along a direction
    d = np.random.default_rng(9).standard_normal(E.shape)
    h = 1e-6
    loss = lambda e: stack_loss(osh, s.cu, None, SCALE * e[s.ids], Ws, gain, e, s.labels)
    measured = (loss(E + h * d) - loss(E - h * d)) / (2 * h)
    # (as the sum of n independent errors within the bar of each element, three times over, and the difference's own of about 1e-8)
    assert abs(measured - float((to_np(raw[-1]) * d).sum())) <= 3 * TOL[dtype] * np.abs(want[-1]).max() * np.sqrt(d.size) + 1e-6


def test_captured_step_replays():
    s = Step("medium", "bf16", [100, 37], 300, 2, 0.05)
    def captured():
        s.gradients()
        s.update()

    eager = []
    for _ in range(3):
        captured()
        eager.append(s.state())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        captured()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured()
    for rep in range(2):
        s.reset()
        for k in range(3):
            graph.replay()
            got = s.state()
            assert all(torch.equal(a, b) for a, b in zip(got, eager[k])), (rep, k)
    assert not torch.equal(eager[0][0], eager[1][0])
