"""The policy loss on tokens that are all but certain, as most of a served response are: the label's gradient is d (1 - p), and what is left of 1
beside p has to keep its digits.

Tolerances: 1 - p = r / (1 + r) with r the sum of the other tokens' exponentials relative to the label's.  r has the relative error E of a
sum of exponentials (u = 2^-24, E = u (2.9 R + 36 + V / 1024), R the distance from the largest logit to those that matter of r: here up to log(V / r) and the
spread of the others), the quotient and the product with d three roundings more.  d = w (-ratio A - c (exp(ref - logp) - 1)) has er = E_logp + 4 u on
either term as in the tests of ordinary rows, with |logp| < 1e-3 here."""
import math

import pytest
import torch

from test_gpu_policy import DT, KL, U, make

pytestmark = pytest.mark.gpu
LEFT = [1e-3, 1e-4, 1e-5, 1e-6, 1e-7, 3e-8, 1e-8, 1e-9, 1e-12, 1e-20]


def peaked(n, V, dtype, seed):
    c = make(n, V, dtype, seed)
    x, m = c["x"], min(n, 2 * len(LEFT))
    spots = [0, V - 1, 3, V // 2, V - 5, 1, V // 3, 8, V - 8, 2]
    for i in range(m):
        at, left = spots[i % len(spots)], LEFT[i % len(LEFT)]
        c["label"][i] = at
        others = torch.cat([x[i, :at], x[i, at + 1:]]).double()
        x[i, at] = (torch.logsumexp(others, 0) - math.log(left)).to(DT[dtype])
    rest, others = terms(c)
    logp = -torch.log1p(rest)
    c["old"][:m], c["ref"][:m] = (logp[:m] + 0.05).float(), (logp[:m] - 0.2).float()
    return c, m


def terms(c):
    """r of every row, in 64 bits, and its terms."""
    x = c["x"].double()
    e = torch.exp(x - x.gather(1, c["label"].long()[:, None]))
    e.scatter_(1, c["label"].long()[:, None], 0.0)
    return e.sum(1), e


# rows of a few hundred bytes to several work-groups' parts, rows of which one stays, rows beyond the registers
@pytest.mark.parametrize("dtype,n,V", [("bf16", 20, 501), ("f32", 20, 501), ("f32", 150, 7001), ("bf16", 20, 128256), ("f32", 20, 128257), ("bf16", 300, 65601),
                                       ("bf16", 400, 128256), ("f32", 300, 40003), ("f32", 340, 80000), ("f32", 340, 131075), ("bf16", 340, 230001)])
def test_label_gradients_keep_their_digits(dtype, n, V):
    import paper_2503_01066_amd as A
    c, m = peaked(n, V, dtype, n + V)
    it = A.PolicyItems(c["label"], c["old"], c["adv"], c["weight"], ref_logp=c["ref"])
    loss, logp, dx = A.alch_policy_loss(c["x"], it, kl_coef=KL)
    alone = A.alch_policy_loss(c["x"], it, kl_coef=KL, want_grad=False)[1]
    torch.cuda.synchronize()
    rest, others = (t[:m] for t in terms(c))
    left = rest / (1 + rest)
    w, adv, old, ref = (c[k][:m].double() for k in ("weight", "adv", "old", "ref"))
    want_logp = -torch.log1p(rest)
    R = torch.log(V / rest) + 20
    E = U * (2.9 * R + 36 + V / 1024)
    for got in (logp, alone):
        assert bool(((got[:m].double() - want_logp).abs() <= 2 * E * want_logp.abs()).all()), ((got[:m].double() - want_logp) / want_logp)
    surrogate, kl = w * torch.exp(want_logp - old) * adv, w * KL * torch.expm1(ref - want_logp)  # (ratios of e^-0.05: no bound is met)
    d = -surrogate - kl
    er = E + 8 * U
    ed = (surrogate.abs() + w * KL * torch.exp(ref - want_logp)) * er
    want = d * left
    label = c["label"][:m].long()[:, None]
    own = dx[:m].gather(1, label)[:, 0].double()
    bound = (want.abs() * (2 * E + 8 * U) + ed * left) * (1 + torch.finfo(DT[dtype]).eps) + torch.finfo(DT[dtype]).eps / 2 * want.abs()
    assert bool(((own - want).abs() <= bound).all()), ((own - want) / want, bound / want.abs())
    if dtype == "f32":  # and a row's gradient sums to zero, measured by what its label has
        total = dx[:m].double().sum(1)
        assert bool((total.abs() <= d.abs() * left * (4 * E + 16 * U)).all()), total / (d * left)


def test_certain_tokens_of_a_certain_row():
    """All others forbidden: p = 1, log-probability and gradient are 0 and not merely small."""
    import paper_2503_01066_amd as A
    for n, V in ((3, 5000), (300, 2000), (3, 128256), (300, 70000)):
        c = make(n, V, "bf16", 3)
        keep = c["x"].gather(1, c["label"].long()[:, None])
        c["x"].fill_(-math.inf).scatter_(1, c["label"].long()[:, None], keep)
        c["old"].fill_(0.01), c["ref"].fill_(-0.1)
        it = A.PolicyItems(c["label"], c["old"], c["adv"], c["weight"], ref_logp=c["ref"])
        for grad in (True, False):
            _, logp, dx = A.alch_policy_loss(c["x"], it, kl_coef=KL, want_grad=grad)
            assert bool((logp == 0).all()) and (dx is None or bool((dx == 0).all()))
