"""AdamW with moments in 8 bits where eps is (near) no normal number of fp32: elements without a gradient so far divide 0 by it."""
import numpy as np
import pytest
import torch

from test_gpu_adamw8 import DT, HYPER, U, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,master", [("f32", False), ("f32", True), ("bf16", False), ("bf16", True)])
@pytest.mark.parametrize("eps", [1e-44, 1e-40, 1e-38, 1.2e-38, 1e-30])
def test_zero_over_the_smallest_eps(dtype, master, eps):
    """0 / eps is 0, as in the update with fp32 moments.  The one gradient of 1 has m / sqrt(v) = 1 (step 1): the weight moves by lr, and is rounded once."""
    import paper_2503_01066_amd as A
    w = torch.randn(300, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    before = [w.to(DT[dtype]), torch.zeros(300, dtype=DT[dtype], device="cuda"), w.clone() if master else None]
    before[1][7] = 1.0
    plain, after = ([None if x is None else x.clone() for x in before] for _ in range(2))
    zeros = (np.zeros(300, np.uint8), np.zeros(5, np.uint8))
    run(A, [after], [(zeros, zeros)], [0.0], step=1, **dict(HYPER, eps=eps))
    moments = [torch.zeros(300, device="cuda") for _ in range(2)]
    A.alch_adamw_step(A.AdamwList([plain[0]], [plain[1]], [moments[0]], [moments[1]], masters=[plain[2]] if master else None), step=1, **dict(HYPER, eps=eps))
    rest = torch.arange(300, device="cuda") != 7
    for k in (0, 2):
        if before[k] is not None:
            assert torch.equal(after[k][rest], before[k][rest]) and torch.equal(plain[k][rest], before[k][rest])
            want, bits = before[k][7].double() - HYPER["lr"], torch.finfo(before[k].dtype).eps / 2
            assert abs(after[k][7].double() - want) <= bits * (abs(want) + 1e-3) + 16 * U * HYPER["lr"]
