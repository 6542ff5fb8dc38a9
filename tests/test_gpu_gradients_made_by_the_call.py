"""Gradients that a backward call makes itself and adds to: those of a call that writes them."""
import numpy as np
import pytest
import torch

import synth_inputs as synth
from helpers import TORCH_DT, alch_shape, to_dev
from test_gpu_stack import REC, make_stack

pytestmark = pytest.mark.gpu


def used_memory():
    """Memory whose next owner finds NaN in it."""
    for n in (64, 512, 4096, 60000, 600000, 3000000):
        blocks = [torch.full((n,), float("nan"), device="cuda") for _ in range(8)]
        del blocks


@pytest.mark.parametrize("dtype,shape_name,lens,V", [("f32", "tiny", [5, 1, 0, 8], 53), ("bf16", "medium", [60, 37], 300)])
def test_stack_and_layer_without_tensors_of_the_caller(dtype, shape_name, lens, V):
    import paper_2503_01066_amd as A
    cu = synth.ragged_cu(lens)
    shp, _, Ws, recs, Xf, gf, Wlm, labels = make_stack(shape_name, dtype, cu, 2, V, 1, 0.05)
    shape, batch = alch_shape(shp, dtype), A.Batch(cu)
    dWs = [{k: to_dev(v, dtype) for k, v in W.items()} for W in Ws]
    drecs = [dict({k: to_dev(r[k], dtype) for k in REC}, LSE=torch.from_numpy(r["LSE"]).cuda()) for r in recs]
    dev = [to_dev(x, dtype) for x in (Xf, gf, Wlm)] + [torch.from_numpy(labels).cuda()]
    lora = [{"q": tuple(to_dev(0.1 * np.random.default_rng(l).standard_normal(s).astype(np.float32), dtype) for s in ((8, shp["hidden"]), (shp["n_q_heads"] * shp["head_dim"], 8)))}
            for l in range(2)]
    calls = [lambda **kw: A.alch_stack_backward(shape, batch, drecs, dWs, *dev, **kw),
             lambda **kw: A.alch_stack_backward_lora(shape, batch, drecs, dWs, lora, 8, 2.0, *dev, want=("Wq", "g1"), want_head=True, **kw),
             lambda **kw: A.alch_layer_backward(shape, batch, drecs[0], dWs[0], dev[0], **kw)]
    flat = lambda out: [out[k] for k in sorted(out) if torch.is_tensor(out[k])] + [d[k] for d in out.get("layers", []) for k in sorted(d)]
    half = torch.finfo(TORCH_DT[dtype]).eps / 2
    for call in calls:
        written = flat(call())
        used_memory()
        for stream in (None, torch.cuda.Stream()):
            torch.cuda.synchronize()
            added = flat(call(accumulate=True, stream=stream))
            torch.cuda.synchronize()
            assert len(added) == len(written) >= 4
            for a, b in zip(added, written):
                # (0 + x: one rounding of the same sum, taken in another order perhaps where a product is cut: 2^-24 of its largest terms)
                assert bool(((a.double() - b.double()).abs() <= 2 * half * b.double().abs() + 2.0 ** -18 * b.double().abs().max()).all())
