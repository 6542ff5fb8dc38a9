"""The policy loss of as many items as 32 bits count."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("grad", [True, False])
def test_most_items(grad):
    """Two logits of 0 each, 2^31 - 1 items of which a few score: log-probability -ln 2, ratio 1, gradient -A w (1/2, -1/2)."""
    import paper_2503_01066_amd as A
    n = (1 << 31) - 1
    if torch.cuda.mem_get_info()[0] < 90 << 30:
        pytest.skip("needs 90 GB of device memory")
    x = torch.zeros((n, 2), dtype=torch.bfloat16, device="cuda")
    label = torch.ones(n, dtype=torch.int32, device="cuda")
    weight, logp = torch.zeros(n, device="cuda"), torch.full((n,), 9.0, device="cuda")
    old, advantage = torch.full((n,), -math.log(2), device="cuda"), torch.ones(n, device="cuda")
    at = [0, 77, 1 << 20, (1 << 30) + 5, n - (1 << 18) - 1, n - (1 << 18), n - 1024, n - 1]
    for i, m in enumerate(at):
        weight[m] = float(1 << i)
    loss, _, dx = A.alch_policy_loss(x, A.PolicyItems(label, old, advantage, weight), want_grad=grad, dlogits=x if grad else None, logp=logp)
    torch.cuda.synchronize()
    # each ratio is exp of the difference of two roundings of -ln 2: 2^-24 off at most, the sum rounded once
    assert abs(loss[0].item() + 255.0) <= 255 * 2 ** -22 and loss[3].item() == 0
    for i, m in enumerate(at):
        assert abs(logp[m].item() + math.log(2)) <= 2 ** -23, m
        if grad:
            want = 0.5 * (1 << i)
            assert abs(dx[m, 0].item() - want) <= want * 2 ** -8 and abs(dx[m, 1].item() + want) <= want * 2 ** -8, m
    for b in range(0, n, 1 << 28):  # and nothing of the others, nor left out
        part = logp[b:b + (1 << 28)]
        assert int((part != 0).sum()) == sum(b <= m < b + (1 << 28) for m in at)
        if grad:
            assert int((dx[b:b + (1 << 28)] != 0).any(1).sum()) == sum(b <= m < b + (1 << 28) for m in at)
