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


@pytest.mark.parametrize("H", [64, 4])
def test_rows_times_one_are_copies(H):
    """Every bf16 there is, subnormal ones among them; a signalling NaN comes out quiet, with the rest of its bits."""
    import paper_2503_01066_amd as A
    W = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).cuda().view(-1, H)
    X = A.alch_embed_forward(torch.arange(W.shape[0], dtype=torch.int32, device="cuda"), W)
    quiet = torch.where(torch.isnan(W), torch.full_like(W, 1.0).view(torch.int16) * 0 + 0x40, torch.zeros_like(W.view(torch.int16)))
    assert torch.equal(X.view(torch.int16), W.view(torch.int16) | quiet)
