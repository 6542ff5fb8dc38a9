"""Adapters under the policy loss: head, then adapted layers, against the oracle in 64 bits.
Bar: per output tensor max|gpu - oracle| / max|oracle| <= 2e-2 (bf16) / 1e-4 (f32), as the stack with adapters under the cross-entropy."""
import numpy as np
import pytest
import torch

import synth_inputs as synth
from helpers import TOL, alch_shape, f64, oracle_shape, rel_err, to_dev, to_np
from oracle import WEIGHT_KEYS
from oracle.lora import layer_backward_reuse_lora, stack_forward_lora
from oracle.policy import policy_head
from test_gpu_policy_stack import HIGH, KL, LOW, items_of, scored

pytestmark = pytest.mark.gpu
REC = ("X", "X2", "Q", "K", "V", "O", "G", "U")


@pytest.mark.parametrize("trained", [False, True])
@pytest.mark.parametrize("dtype,shape_name,lens,V,std", [("f32", "tiny", [5, 0, 3, 1], 37, 0.3), ("bf16", "medium", [129, 40, 1, 77], 512, 0.05),
                                                         ("bf16", "medium64", [90, 61], 333, 0.05)])
def test_adapter_gradients_match_the_oracle(dtype, shape_name, lens, V, std, trained):
    import paper_2503_01066_amd as A
    cu, shp, L, rank, scale = synth.ragged_cu(lens), synth.shape_dict(shape_name), 2, 8, 2.0
    osh, T, r = oracle_shape(shp), int(cu[-1]), np.random.default_rng(21)
    Ws = [synth.layer_weights(shp, 40 + 10 * l, dtype, std=std, gain_std=0.1) for l in range(L)]
    loras = [synth.lora_adapters(shp, rank, 90 + l, dtype, ("q", "v") if l == 0 else synth.PROJECTIONS, std=0.1) for l in range(L)]
    X0 = synth.normal(r, (T, shp["hidden"]), 1.0, dtype)
    gf = synth.quantize(1.0 + 0.1 * r.standard_normal(shp["hidden"]).astype(np.float32), dtype)
    Wlm = synth.normal(r, (V, shp["hidden"]), std, dtype)
    loras64 = [{p: (a.astype(np.float64), b.astype(np.float64)) for p, (a, b) in lo.items()} for lo in loras]
    Xf, recs = stack_forward_lora(osh, cu, None, X0.astype(np.float64), [f64(W) for W in Ws], loras64, scale)
    recs = [dict({k: synth.quantize(rec[k].astype(np.float32), dtype) for k in REC}, LSE=rec["LSE"].astype(np.float32)) for rec in recs]
    Xf = synth.quantize(Xf.astype(np.float32), dtype)
    # two thirds of the rows score, some of them twice, some items not at all
    rows = np.sort(np.concatenate([r.permutation(T)[:max(2 * T // 3, 1)], r.integers(0, T, max(T // 8, 1))])).astype(np.int32)
    rows = rows[:T]
    labels = r.integers(0, V, len(rows)).astype(np.int32)
    extra = scored(osh, Xf, gf, Wlm, rows, labels, 5)
    labels[:1] = -1
    loss, dX, dg, dW, logp = policy_head(osh, Xf, gf, Wlm, rows, labels, *extra, LOW, HIGH, KL)
    want = [None] * L
    for l in range(L - 1, -1, -1):
        want[l] = layer_backward_reuse_lora(osh, cu, None, f64(recs[l]), f64(Ws[l]), loras64[l], scale, dX)
        dX = want[l]["dX"]

    records = [dict({k: to_dev(rec[k], dtype) for k in REC}, LSE=torch.from_numpy(rec["LSE"]).cuda()) for rec in recs]
    out = A.alch_stack_backward_policy(alch_shape(shp, dtype), A.Batch(cu), records, [{k: to_dev(v, dtype) for k, v in W.items()} for W in Ws], to_dev(Xf, dtype),
                                       to_dev(gf, dtype), to_dev(Wlm, dtype), items_of(A, rows, labels, *extra), clip_low=LOW, clip_high=HIGH, kl_coef=KL,
                                       lora_layers=[{p: (to_dev(a, dtype), to_dev(b, dtype)) for p, (a, b) in lo.items()} for lo in loras], rank=rank, scale=scale,
                                       **({} if trained else dict(want=(), want_head=False)))
    torch.cuda.synchronize()
    tol = TOL[dtype]
    assert np.abs(to_np(out["logp"]) - logp).max() <= tol * max(1.0, np.abs(logp).max()) and np.abs(to_np(out["loss"]) - loss).max() <= tol * max(1.0, np.abs(loss).max())
    errors = {"dX_embed": rel_err(to_np(out["dX_embed"]), dX)}
    if trained:
        errors.update(dg_final=rel_err(to_np(out["dg_final"]), dg), dW_lm=rel_err(to_np(out["dW_lm"]), dW))
    else:
        assert out["dg_final"] is None and out["dW_lm"] is None
    for l in range(L):
        keys = ["d" + m + p for p in loras[l] for m in "AB"] + (["d" + k for k in WEIGHT_KEYS] if trained else [])
        assert sorted(out["layers"][l]) == sorted(keys)
        errors.update({(l, k): rel_err(to_np(out["layers"][l][k]), want[l][k]) for k in keys})
    assert max(errors.values()) <= tol, errors
