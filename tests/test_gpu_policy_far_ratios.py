"""The policy loss where the policies are far from each other: ratios and exp(ref - logp) beyond fp32, and labels that the logits forbid.

An entry of the gradient is -d p (the label's d (1 - p)), a number of 64 bits rounded once: infinite where it is beyond the storage type, 0 where
the logit is -inf, whatever d is.  Tolerances: an exponential exp(a) with a rounded to fp32 is off by |a| 2^-24 relative, a of size F = logp - old or
ref - logp; the rest as in the tests of ordinary rows."""
import math

import pytest
import torch

from test_gpu_policy import DT, U, formula, make

pytestmark = pytest.mark.gpu
SIZES = [("f32", 5, 1001), ("bf16", 5, 1001), ("f32", 200, 3000), ("bf16", 9, 128256), ("f32", 9, 40001), ("bf16", 300, 70000), ("f32", 300, 40000), ("f32", 340, 120000)]


def run(A, c, kl, grad=True, **kw):
    it = A.PolicyItems(c["label"], c["old"], c["adv"], c["weight"], ref_logp=c["ref"])
    out = A.alch_policy_loss(c["x"], it, kl_coef=kl, want_grad=grad, **kw)
    torch.cuda.synchronize()
    return out


def half_forbidden(n, V, dtype):
    c = make(n, V, dtype, n + V)
    keep = c["x"].gather(1, c["label"].long()[:, None])
    c["x"][:, ::2] = -math.inf
    c["x"].scatter_(1, c["label"].long()[:, None], keep)
    c["weight"].fill_(1.0)
    logp = torch.log_softmax(c["x"].double(), 1).gather(1, c["label"].long()[:, None])[:, 0]
    c["old"], c["ref"] = (logp + 0.05).float(), (logp - 0.1).float()
    return c, logp


@pytest.mark.parametrize("dtype,n,V", SIZES)
@pytest.mark.parametrize("what", ["ref", "ratio", "both", "weighted"])
def test_slopes_beyond_fp32(dtype, n, V, what):
    import paper_2503_01066_amd as A
    c, logp = half_forbidden(n, V, dtype)
    kl = 0.07
    far = torch.linspace(60.0, 180.0, n, device="cuda", dtype=torch.float64)
    if what in ("ref", "both", "weighted"):
        c["ref"] = (logp + far).float()
    if what in ("ratio", "both"):
        c["adv"] = -c["adv"].abs() - 0.1  # (a ratio above the bound counts where the advantage is negative)
        c["old"] = (logp - far.flip(0)).float()
    if what == "weighted":
        c["weight"] = torch.exp(-far).float().clamp(min=1e-37)
    loss, got_logp, dx = run(A, c, kl)
    want, _, wdx, t = formula(**c, kl_coef=kl, low=0.2, high=0.2)
    assert not bool(torch.isnan(dx).any()) and bool((dx[torch.isneginf(c["x"])] == 0).all())
    big = torch.finfo(DT[dtype]).max
    E = U * (2.9 * t["R"] + 36 + V / 1024)
    rel = 2 * E + 3 * U * (logp.abs() + t["R"] + t["logz"].abs()) + 200 * U * 2 + 24 * U + torch.finfo(DT[dtype]).eps / 2
    over, under = wdx.abs() > big * (1 + 2 ** -7), wdx.abs() < big * (1 - 2 ** -7)
    assert bool((torch.isinf(dx) & (dx.double().sign() == wdx.sign()))[over].all())
    off = (dx.double() - wdx).abs()
    # a surrogate and a KL term of opposite signs leave less than either: their errors count by their own size, times p or 1 - p
    size = torch.maximum(wdx.abs(), ((t["w"] * (t["ratio"] + t["kl"])).clamp(max=1e300)[:, None] * t["p"]))
    size.scatter_(1, c["label"].long()[:, None], (t["w"] * (t["ratio"] + t["kl"]) + t["d"].abs())[:, None])
    bound = rel[:, None] * size + 2e-38 * (1 if dtype == "bf16" else 2 ** -20)
    assert not bool(((off > bound) & under).any()), torch.nonzero((off > bound) & under)[:4]
    finite = want.abs() < 3e38
    assert bool(torch.isinf(loss[:3].double())[~finite[:3]].all()) and not bool(torch.isnan(loss).any())
    alone = run(A, c, kl, grad=False)[0]
    for l in (loss, alone):
        assert bool(((l.double() - want).abs() <= 400 * U * want.abs() + 1e-30)[finite].all()), (l, want)


@pytest.mark.parametrize("dtype,n,V", SIZES)
def test_labels_that_the_logits_forbid(dtype, n, V):
    """logp = -inf: the ratio is 0, the KL term infinite.  Its gradient is infinite where tokens are allowed and 0 where they are not, the label among them;
    without a coefficient the term is measured and adds nothing."""
    import paper_2503_01066_amd as A
    c, _ = half_forbidden(n, V, dtype)
    c["x"][1].scatter_(0, c["label"][1:2].long(), -math.inf)
    for grad in (True, False):
        loss, logp, dx = run(A, c, 0.0, grad)
        assert logp[1].item() == -math.inf and bool(torch.isfinite(logp[torch.arange(n) != 1]).all())
        assert math.isfinite(loss[0].item()) and loss[0] == loss[1] and loss[2].item() == math.inf and math.isfinite(loss[3].item())
        assert dx is None or bool((dx[1] == 0).all()) and bool(torch.isfinite(dx).all())
        loss, logp, dx = run(A, c, 0.1, grad)
        assert logp[1].item() == -math.inf and loss[0].item() == math.inf and loss[2].item() == math.inf and math.isfinite(loss[1].item())
        if grad:
            assert not bool(torch.isnan(dx).any()) and bool((dx[torch.isneginf(c["x"])] == 0).all())
            p = torch.softmax(c["x"][1].double(), 0)
            assert bool((dx[1][p > 1e-30] == math.inf).all())
            rows = torch.arange(n, device="cuda") != 1
            assert bool(torch.isfinite(dx[rows]).all())
    # the reference model forbids what the policy allows: log-ratio -inf, the KL term infinite, its gradient the plain coefficient
    c, logp = half_forbidden(n, V, dtype)
    c["ref"][1] = -math.inf
    c["adv"][1] = 0.0
    loss, _, dx = run(A, c, 0.25)
    p = torch.softmax(c["x"][1].double(), 0)
    want = -0.25 * p
    want[c["label"][1].long()] += 0.25
    assert loss[2].item() == math.inf and bool(torch.isfinite(dx).all())
    assert float((dx[1].double() - want).abs().max()) <= 0.25 * (torch.finfo(DT[dtype]).eps / 2 + 1e-4)
