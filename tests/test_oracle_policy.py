"""The oracle of the policy loss: finite differences of its loss, closed forms at the reference policy, items that score nothing."""
import numpy as np

from oracle import LayerShape
from oracle.policy import policy_head

SHAPE = LayerShape(16, 4, 2, 4, 24, 1e-6, 10000.0)


def case(seed, n=9, V=23):
    r = np.random.default_rng(seed)
    X, g, W = r.normal(size=(7, 16)), 1 + 0.1 * r.normal(size=16), 0.4 * r.normal(size=(V, 16))
    rows = np.sort(r.integers(0, 7, n))
    label = r.integers(0, V, n)
    logp = policy_head(SHAPE, X, g, W, rows, label, np.zeros(n), np.zeros(n), np.ones(n), None, 0.2, 0.2, 0.0)[4]
    return [X, g, W], [rows, label, logp - r.choice([-0.4, -0.1, 0.05, 0.1, 0.4], n), r.normal(size=n), r.uniform(0.1, 1, n), logp + 0.3 * r.normal(size=n)]


def test_finite_differences():
    P, items = case(1)
    loss, dX, dg, dW, _ = policy_head(SHAPE, *P, *items, 0.2, 0.3, 0.07)
    assert loss[3] > 0 and loss[2] > 0
    r, h = np.random.default_rng(2), 1e-6
    for k, grad in enumerate((dX, dg, dW)):
        way = r.normal(size=P[k].shape)
        at = lambda s: policy_head(SHAPE, *[p + s * h * way if i == k else p for i, p in enumerate(P)], *items, 0.2, 0.3, 0.07)[0][0]
        assert abs((at(1) - at(-1)) / (2 * h) - (grad * way).sum()) <= 1e-7 * np.abs(grad * way).sum()


def test_closed_forms():
    P, items = case(3)
    rows, label, old, adv, w, ref = items
    logp = policy_head(SHAPE, *P, *items, 0.2, 0.2, 0.0)[4]
    # at the sampling policy the loss is -sum w A, with the gradient of -sum w A logp; at the reference the KL term is flat
    a = policy_head(SHAPE, *P, rows, label, logp, adv, w, logp, 0.2, 0.2, 3.0)
    assert np.allclose(a[0], [-(w * adv).sum(), -(w * adv).sum(), 0, 0], atol=1e-12)
    b = policy_head(SHAPE, *P, rows, label, logp, adv, w, None, np.inf, np.inf, 0.0)
    assert all(np.allclose(x, y, atol=1e-12) for x, y in zip(a[1:4], b[1:4]))


def test_items_that_score_nothing():
    P, (rows, label, old, adv, w, ref) = case(4)
    less = [0, 2, 5]
    label2, w2 = label.copy(), w.copy()
    label2[1], label2[3], w2[[4, 6, 7, 8]] = -1, 23, 0
    a = policy_head(SHAPE, *P, rows, label2, old, adv, w2, ref, 0.2, 0.2, 0.1)
    b = policy_head(SHAPE, *P, *[x[less] for x in (rows, label, old, adv, w, ref)], 0.2, 0.2, 0.1)
    assert all(np.allclose(x, y, atol=1e-12) for x, y in zip(a[:4], b[:4]))
    assert (a[4][[1, 3, 4, 6, 7, 8]] == 0).all()
