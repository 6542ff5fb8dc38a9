"""Batches of many sizes in one workspace, made for the largest of them."""
import numpy as np
import pytest
import torch

from test_gpu_embed import check_backward, make_ids, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H,V,sizes", [(4096, 3000, (16384, 16000, 8192, 8176, 4090, 500, 1)), (72, 40000, (270000, 262144, 262145, 65000, 8000)),
                                       (8200, 9000, (7711, 7710, 3856, 3855, 2100))])
def test_smaller_batches_in_the_workspace_of_the_largest(H, V, sizes):
    import paper_2503_01066_amd as A
    size = A.embed_backward_workspace_bytes(torch.bfloat16, V, H, max(sizes))
    memory = torch.full((size + 4096,), 0x7f, dtype=torch.uint8, device="cuda")
    for n in sizes:
        ids, dX = make_ids("runs", n, V, n), randn((n, H), "bf16", n, 0.01)
        dev, old = (torch.from_numpy(ids).cuda(), dX.cuda()), randn((V, H), "bf16", 5, 0.1)
        dW = A.alch_embed_backward(*dev, V, workspace=memory[:size])
        check_backward(ids, dX, V, 1.0, dW, None)
        dW = A.alch_embed_backward(*dev, V, dW_embed=old.cuda(), accumulate=True, workspace=memory[:size])
        check_backward(ids, dX, V, 1.0, dW, old)
        assert bool((memory[size:] == 0x7f).all())
