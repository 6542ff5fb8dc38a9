"""Oracle for the clipped policy loss with a KL term on sampled tokens, on top of the layer stack.

Test infrastructure only (see the package docstring).  float64 throughout.

The paper's example of preference alignment is DPO (Section 6); here the responses that serving sampled carry an advantage
each, and the loss of an item m with log-probability lp, ratio r = exp(lp - old), advantage A and weight w is
w * (-min(r A, clip(r, 1 - lo, 1 + hi) A) + c * (exp(ref - lp) - (ref - lp) - 1)); the loss is the sum over the items.
Items with a label outside the vocabulary or weight 0 score nothing.
"""
import numpy as np

from .layer import _rms_norm, _rms_norm_backward
from .prefix import layer_backward_reuse_prefix


def policy_head(shape, X_final, g_final, W_lm, item_row, label, old, adv, weight, ref, lo, hi, c):
    """Returns (loss [4] = loss, surrogate, kl, clipped weight; dX_final, dg_final, dW_lm, logp [items])."""
    X_final, g_final, W_lm = (np.asarray(a, dtype=np.float64) for a in (X_final, g_final, W_lm))
    rows, label = np.asarray(item_row, dtype=np.int64), np.asarray(label, dtype=np.int64)
    Hf, rf = _rms_norm(X_final, g_final, shape.rms_eps)
    logits = Hf[rows] @ W_lm.T
    top = logits.max(axis=1, keepdims=True) if len(rows) else np.zeros((0, 1))
    logp_all = logits - top - np.log(np.exp(logits - top).sum(axis=1, keepdims=True))
    dlogits, logp, loss = np.zeros_like(logits), np.zeros(len(rows)), np.zeros(4)
    for m in range(len(rows)):
        if not 0 <= label[m] < W_lm.shape[0] or weight[m] == 0:
            continue
        lp, A, w = logp_all[m, label[m]], float(adv[m]), float(weight[m])
        r = np.exp(lp - old[m])
        bounded = min(max(r, 1 - lo), 1 + hi) * A
        clipped = bounded < r * A
        slope = 0.0 if clipped else -r * A
        kl = 0.0
        if ref is not None:
            gap = ref[m] - lp
            kl = np.exp(gap) - gap - 1
            slope += c * (1 - np.exp(gap))
        loss += w * np.array([-min(r * A, bounded) + c * kl, -min(r * A, bounded), kl, clipped])
        dlogits[m] = -w * slope * np.exp(logp_all[m])
        dlogits[m, label[m]] += w * slope
        logp[m] = lp
    dHf = np.zeros_like(X_final)
    np.add.at(dHf, rows, dlogits @ W_lm)
    dX, dg = _rms_norm_backward(dHf, X_final, g_final, rf)
    return loss, dX, dg, dlogits.T @ Hf[rows], logp


def stack_backward_policy(shape, cu_seqlens, prefix, recs, layers_W, X_final, g_final, W_lm, *items):
    """The head, then the layers from the last to the first, each from its own saved record."""
    loss, dX, dg, dW, logp = policy_head(shape, X_final, g_final, W_lm, *items)
    layers = [None] * len(layers_W)
    for l in range(len(layers_W) - 1, -1, -1):
        layers[l] = layer_backward_reuse_prefix(shape, cu_seqlens, prefix, recs[l], layers_W[l], dX)
        dX = layers[l]["dX"]
    return dict(loss=loss, logp=logp, dX_embed=dX, dg_final=dg, dW_lm=dW, layers=layers)
