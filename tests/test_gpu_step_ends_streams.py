"""Lists made on one stream and used on the current one of a block, then dropped."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_lists_dropped_behind_calls_on_the_current_stream():
    import paper_2503_01066_amd as A
    s = torch.cuda.Stream()
    g = [torch.randn(300000, device="cuda").bfloat16(), torch.randn(77, device="cuda")]
    want = A.alch_grad_clip(A.GradList(g), 1.0)
    torch.cuda.synchronize()
    norms = []
    for _ in range(20):
        grads = A.GradList(g)
        with torch.cuda.stream(s):
            norms.append(A.alch_grad_clip(grads, 1.0))
        del grads
        torch.full((4096,), 0x7f, dtype=torch.uint8, device="cuda")  # (memory that was just freed is written again)
    torch.cuda.synchronize()
    assert all(torch.equal(n, want) for n in norms)


def test_update_by_a_list_dropped_behind_its_call():
    import paper_2503_01066_amd as A
    s = torch.cuda.Stream()
    p, g, m, v = ([torch.randn(n, device="cuda").square() for n in (200000, 9)] for _ in range(4))
    start = [x.clone() for x in p + m + v]
    runs = []
    for stream in (None, s):
        for x, y in zip(p + m + v, start):
            x.copy_(y)
        torch.cuda.synchronize()
        for step in range(1, 4):
            tensors = A.AdamwList(p, g, m, v, weight_decay=0.1)
            with torch.cuda.stream(stream):
                A.alch_adamw_step(tensors, 1e-2, step=step)
            del tensors
            torch.full((4096,), 0x7f, dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        runs.append([x.clone() for x in p + m + v])
    assert all(torch.equal(a, b) for a, b in zip(*runs)) and not torch.equal(runs[0][0], start[0])


def test_a_list_used_by_a_capture_lives_as_long_as_its_graph():
    import paper_2503_01066_amd as A
    g = [torch.randn(5000, device="cuda")]
    norm, ws = torch.empty(2, device="cuda"), torch.empty(A.grad_clip_workspace_bytes(), dtype=torch.uint8, device="cuda")
    grads, graph = A.GradList(g), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        A.alch_grad_clip(grads, 1.0, norm_out=norm, workspace=ws)
    for k in range(3):
        g[0].normal_()
        eager = A.alch_grad_clip(grads, 1.0)
        norm.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(norm, eager)
    del graph, grads
    torch.cuda.synchronize()
    torch.full((4096,), 0x7f, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
