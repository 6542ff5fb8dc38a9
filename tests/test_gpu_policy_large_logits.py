"""The policy loss on logits of about a million: a sum in one pass is scaled by a power of two, and powers are exact up to 2^20 only.  Rows on
either side of that border, and across it, against the formulas in 64 bits with the tolerances of the loss on ordinary rows (differences of such
logits are exact, what is rounded is the same)."""
import pytest
import torch

from test_gpu_policy import KL, check, make

pytestmark = pytest.mark.gpu
BORDER = 1048576.0


def plant(c):
    """Row 0: the largest logit alone stands on the border, row 1 is spread over it, rows 2 to 5 lie just inside and outside of it, 6 and 7 are row 1 far from
    it; each for both signs.  The label is a likely token in all of them."""
    n, V = c["x"].shape
    g = torch.Generator(device="cuda").manual_seed(1)
    spread = lambda: (torch.randn(V, generator=g, device="cuda") * 2)
    rows = []
    for sign in (-1.0, 1.0):
        top = torch.full((V,), sign * BORDER - 1, device="cuda")
        top[V // 3] = sign * BORDER
        rows.append(top)
        rows += [sign * BORDER + at + spread() for at in (0.0, -4.0, 20.0, -130.0, 130.0, 0.5 * BORDER, -0.5 * BORDER)]
    for i, r in enumerate(rows):
        c["x"][i] = r
        c["label"][i] = V // 3 if i % 8 == 0 else int(r.argmax()) if i % 2 else 7
    logp = torch.log_softmax(c["x"][:len(rows)].double() - c["x"][:len(rows)].double().amax(1, keepdim=True), 1)
    logp = logp.gather(1, c["label"][:len(rows)].long()[:, None])[:, 0]
    c["old"][:len(rows)], c["ref"][:len(rows)] = (logp + 0.05).float(), (logp - 0.1).float()
    return c


# 16 whole rows without a gradient and rows in registers with one; rows in parts, short ones and long ones; rows of which the end is read again
@pytest.mark.parametrize("n,V", [(330, 32000), (16, 5000), (200, 150001), (330, 128256)])
@pytest.mark.parametrize("grad", [False, True])
def test_rows_across_the_largest_exact_power(n, V, grad):
    import paper_2503_01066_amd as A
    check(A, plant(make(n, V, "f32", n + V)), kl_coef=KL, grad=grad)


def test_one_logit_on_the_border():
    """32,000 logits: log(1 + 31999 / e) = 9.3735 is what the others take from the largest one."""
    import paper_2503_01066_amd as A
    c = plant(make(330, 32000, "f32", 5))
    it = A.PolicyItems(c["label"], c["old"], c["adv"], c["weight"], ref_logp=c["ref"])
    for grad in (False, True):
        logp = A.alch_policy_loss(c["x"], it, want_grad=grad)[1]
        assert abs(logp[0].item() + 9.3735) <= 1e-4, (grad, logp[0].item())
