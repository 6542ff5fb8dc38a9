"""alch_grad_clip and alch_adamw_step against their definitions in 64 bits.

Tolerances count roundings, u = 2^-24: the norm is summed in 64 bits and rounded once; the factor once; a clipped value has
the factor's, the product's and the storage type's half step.  The update: m has at most four (b1, d1, two products, the sum:
on |b1 m| + |d1 g'|, g' with its own one), v six on a sum of positive terms, the step m c1 / (sqrt(v c2) + eps) those of m and
half of v's, and one each for c1, the product, c2, its product (halved), the root, the sum, the quotient: at most 12; decay, its sum,
the rate and its product four more on the whole change, w the last one."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
U = 2.0 ** -24
SIZES = [0, 1, 7, 8, 9, 255, 2047, 2048, 2049, 8191, 8193, 0, 100003, 3]


def half(t):
    return torch.finfo(t.dtype).eps / 2


def tensors(sizes, dtypes, seed, std=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [(torch.randn(n, generator=g, device="cuda") * std).to(DT[dtypes[i % len(dtypes)]]) for i, n in enumerate(sizes)]


def check_clip(grads, before, outs, norm, max_norm):
    ref = math.sqrt(sum(float(b.double().square().sum()) for b in before))
    factor = max_norm / ref if ref > max_norm else 1.0
    got = norm.tolist()
    assert abs(got[0] - ref) <= 1.01 * U * ref and abs(got[1] - factor) <= 1.01 * U * factor, (got, ref, factor)
    for b, o in zip(before, outs):
        if o is not None:
            want = b.double() * factor
            assert bool(((o.double() - want).abs() <= (2.01 * U + half(b)) * want.abs() + 1e-44).all())
            if factor == 1.0:
                assert torch.equal(o, b)


@pytest.mark.parametrize("dtypes", [["bf16"], ["f32"], ["f32", "bf16", "bf16"]])
@pytest.mark.parametrize("max_norm", [1.0, 1e6, 0.0, math.inf])
def test_clip(dtypes, max_norm):
    import paper_2503_01066_amd as A
    grads = tensors(SIZES, dtypes, 1)
    before = [g.clone() for g in grads]
    outs = [torch.full_like(g, 9.0) for g in grads]
    norm = A.alch_grad_clip(A.GradList(grads, outs), max_norm)
    check_clip(grads, before, outs, norm, max_norm)
    assert all(torch.equal(a, b) for a, b in zip(grads, before))
    # in place, every third tensor counted only, whatever the workspace held
    place = [None if i % 3 == 2 else g for i, g in enumerate(grads)]
    ws = torch.full((A.grad_clip_workspace_bytes(),), 0xff, dtype=torch.uint8, device="cuda")
    norm2 = A.alch_grad_clip(A.GradList(grads, place), max_norm, workspace=ws)
    check_clip(grads, before, place, norm2, max_norm)
    assert torch.equal(norm, norm2)
    assert all(torch.equal(g, b) for i, (g, b) in enumerate(zip(grads, before)) if i % 3 == 2)
    for g, b in zip(grads, before):
        g.copy_(b)
    only = A.alch_grad_clip(A.GradList(grads), max_norm)
    assert torch.equal(only, norm) and all(torch.equal(a, b) for a, b in zip(grads, before))


def test_clip_leaves_what_lies_between_the_tensors():
    import paper_2503_01066_amd as A
    flat = torch.randn(4096 * 4, device="cuda").bfloat16()
    cuts = [(0, 5), (8, 1), (16, 4091), (4112, 8192)]
    old = flat.clone()
    views = [flat[a:a + n] for a, n in cuts]
    A.alch_grad_clip(A.GradList(views, views), 0.5)
    inside = torch.zeros(flat.numel(), dtype=torch.bool, device="cuda")
    for a, n in cuts:
        inside[a:a + n] = True
    assert torch.equal(flat[~inside], old[~inside]) and not torch.equal(flat[inside], old[inside])


def test_clip_of_many_tensors_and_of_none():
    import paper_2503_01066_amd as A
    r = np.random.default_rng(0)
    for n in (63, 64, 65, 257, 4096):
        grads = tensors(r.integers(0, 40, n).tolist(), ["f32", "bf16"], n)
        before = [g.clone() for g in grads]
        norm = A.alch_grad_clip(A.GradList(grads, grads), 2.0)
        check_clip(grads, before, grads, norm, 2.0)
    assert A.alch_grad_clip(A.GradList([]), 1.0).tolist() == [0.0, 1.0]
    assert A.alch_grad_clip(A.GradList([torch.empty(0, device="cuda")] * 3), 0.0).tolist() == [0.0, 1.0]
    with pytest.raises(A.AlchError, match="4096"):
        A.alch_grad_clip(A.GradList([torch.zeros(1, device="cuda")] * 4097), 1.0)


def test_norms_whose_squares_leave_32_bits():
    import paper_2503_01066_amd as A
    for size in (1e30, 1e-30):
        g = [torch.full((5000,), size, device="cuda"), torch.full((77,), size, device="cuda").bfloat16()]
        norm = A.alch_grad_clip(A.GradList(g), size)
        ref = math.sqrt(sum(float(x.double().square().sum()) for x in g))
        assert abs(norm[0].item() - ref) <= 1.01 * U * ref and abs(norm[1].item() - float(np.float32(size)) / ref) <= 2 * U * size / ref


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_norm_that_is_no_number(bad):
    import paper_2503_01066_amd as A
    g = tensors([100, 5000, 9], ["bf16"], 3)
    g[1][4321] = bad
    p, m, v, w = [[torch.randn(x.numel(), device="cuda") for x in g] for _ in range(4)]
    p = [x.bfloat16() for x in p]
    norm = A.alch_grad_clip(A.GradList(g, g), 1.0)
    assert not math.isfinite(norm[0].item()) and math.isnan(norm[1].item())
    assert all(bool(torch.isnan(x).all()) for x in g)
    old = [x.clone() for x in p + m + v + w]
    for f in (norm[1:], torch.full((1,), math.inf, device="cuda")):
        A.alch_adamw_step(A.AdamwList(p, g, m, [x.abs_() for x in v], masters=w), 0.1, grad_factor=f)
    assert all(torch.equal(a, b) for a, b in zip(p + m + w, old[:6] + old[9:]))
    assert all(torch.equal(a, b.abs()) for a, b in zip(v, old[6:9]))


def adamw_reference(p, g, m, v, w, decay, f, lr, b1, b2, eps, step):
    """(new w, m, v in 64 bits, their bounds)"""
    old = (p if w is None else w).double()
    x = g.double() * f
    a, b = b1 * m.double(), (1 - b1) * x
    nm, nv = a + b, b2 * v.double() + (1 - b2) * x.square()
    em = 5 * U * (a.abs() + b.abs()) + 1e-44
    c1, den = 1 / (1 - b1 ** step), (nv / (1 - b2 ** step)).sqrt() + eps
    change = nm * c1 / den
    nw = old - lr * (change + decay * old)
    ew = lr * (em * c1 / den + 16 * U * change.abs() + 6 * U * (decay * old).abs()) + U * (nw.abs() + lr * (change + decay * old).abs()) + 1e-44
    return nw, nm, nv, ew, em, 8 * U * nv + 1e-44


@pytest.mark.parametrize("dtype,master", [("f32", False), ("bf16", False), ("bf16", True), ("f32", True)])
@pytest.mark.parametrize("step,factor", [(1, None), (7, 0.25), (100000, 1.0)])
def test_adamw(dtype, master, step, factor):
    import paper_2503_01066_amd as A
    hyper = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=step)
    p, g = tensors(SIZES, [dtype], 1), tensors(SIZES, [dtype], 2, 0.01)
    g[6][:100] = 0.0
    m, v = tensors(SIZES, ["f32"], 3, 0.005 if step > 1 else 0.0), [x.square() for x in tensors(SIZES, ["f32"], 4, 0.01 if step > 1 else 0.0)]
    w = [x.float() + 1e-4 * torch.randn_like(x.float()) for x in p] if master else [None] * len(p)
    decay = [0.1 if i % 2 else 0.0 for i in range(len(p))]
    fac = None if factor is None else torch.full((1,), factor, device="cuda")
    ref = [adamw_reference(*t, f=1.0 if factor is None else factor, lr=1e-3, b1=0.9, b2=0.999, eps=1e-8, step=step)
           for t in zip(p, g, m, v, w, [float(np.float32(d)) for d in decay])]
    A.alch_adamw_step(A.AdamwList(p, g, m, v, masters=w if master else None, weight_decay=decay), grad_factor=fac, **hyper)
    for i, (nw, nm, nv, ew, em, ev) in enumerate(ref):
        for name, got, want, bound in (("m", m[i], nm, em), ("v", v[i], nv, ev), ("w", w[i] if master else p[i], nw, ew)):
            bound = bound + (half(got) * (want.abs() + bound) if got.dtype != torch.float32 else 0)
            err = (got.double() - want).abs()
            assert bool((err <= bound).all()), (i, name, float((err / bound).max()))
        if master:
            assert torch.equal(p[i], w[i].to(p[i].dtype))


def test_adamw_schedule_on_the_device_is_the_same_update():
    import paper_2503_01066_amd as A
    start = [tensors([5000, 37], ["bf16"], 1), tensors([5000, 37], ["bf16"], 2), tensors([5000, 37], ["f32"], 3), [x.square() for x in tensors([5000, 37], ["f32"], 4)]]
    out = []
    for schedule in (None, torch.tensor([3e-4, 12.0], device="cuda")):
        p, g, m, v = [[x.clone() for x in l] for l in start]
        w = [x.float() for x in p]
        A.alch_adamw_step(A.AdamwList(p, g, m, v, masters=w), 3e-4 if schedule is None else 99.0, step=12 if schedule is None else 1, schedule=schedule)
        out.append(w + m + v + p)
    # (the powers are taken on the host and on the device: up to one rounding of each correction)
    for a, b in zip(*out):
        assert bool(((a - b).abs().double() <= 2 * (half(a) + 4 * U) * b.abs().double()).all())


@pytest.mark.parametrize("step", [0.0, -1.0, math.nan])
def test_adamw_schedule_that_is_no_step_changes_nothing(step):
    import paper_2503_01066_amd as A
    p, g, m, v = (tensors([5000, 3], ["f32"], k) for k in range(4))
    old = [x.clone() for x in p + m + v]
    A.alch_adamw_step(A.AdamwList(p, g, m, v), 1.0, schedule=torch.tensor([1.0, step], device="cuda"))
    assert all(torch.equal(a, b) for a, b in zip(p + m + v, old))


def test_lists_dropped_behind_calls_on_another_stream():
    import paper_2503_01066_amd as A
    s = torch.cuda.Stream()
    g = tensors([300000, 77], ["bf16"], 1)
    want = A.alch_grad_clip(A.GradList(g), 1.0)
    torch.cuda.synchronize()
    norms = []
    for _ in range(20):
        norms.append(A.alch_grad_clip(A.GradList(g), 1.0, stream=s))
        torch.full((4096,), 0x7f, dtype=torch.uint8, device="cuda")  # (memory that was just freed is written again)
    torch.cuda.synchronize()
    assert all(torch.equal(n, want) for n in norms)


def test_captured_step_follows_its_schedule_and_gradients():
    import paper_2503_01066_amd as A
    sizes = [3000, 9, 70000]
    g, p = tensors(sizes, ["bf16"], 2), tensors(sizes, ["bf16"], 1)
    state = lambda: [x.float() for x in p] + [torch.zeros(n, device="cuda") for n in sizes * 2]
    runs = []
    grads, params, s = [x.clone() for x in g], [x.clone() for x in p], state()
    norm, ws = torch.empty(2, device="cuda"), torch.empty(A.grad_clip_workspace_bytes(), dtype=torch.uint8, device="cuda")
    schedule = torch.zeros(2, device="cuda")
    clip, opt = A.GradList(grads), A.AdamwList(params, grads, s[3:6], s[6:], masters=s[:3], weight_decay=0.01)

    def step():
        A.alch_grad_clip(clip, 1.0, norm_out=norm, workspace=ws)
        A.alch_adamw_step(opt, 0.0, schedule=schedule, grad_factor=norm[1:])

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for how in (step, graph.replay):
        for x, y in zip(params + s, p + state()):
            x.copy_(y)
        got = []
        for k in range(1, 4):
            for x, y in zip(grads, g):
                x.copy_(y * k)
            schedule.copy_(torch.tensor([1e-2 / k, float(k)]))
            torch.cuda.synchronize()
            how()
            torch.cuda.synchronize()
            got.append([x.clone() for x in params + s + [norm]])
        runs.append(got)
    for a, b in zip(*runs):
        assert all(torch.equal(x, y) for x, y in zip(a, b))
    assert not torch.equal(runs[0][0][0], runs[0][1][0])


def test_tensors_beyond_32_bit_offsets():
    import paper_2503_01066_amd as A
    n = (1 << 31) + 12345  # elements, 4.3 GB in bf16
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g[n - 3:] = 2.0
    g[5] = 2.0
    norm = A.alch_grad_clip(A.GradList([g, g], [None, None]), 1.0)  # (twice in the list, only read)
    assert abs(norm[0].item() - math.sqrt(32)) <= 1e-6
    A.alch_grad_clip(A.GradList([g], [g]), 1.0)
    assert g[n - 4:].tolist() == [0.0, 0.5, 0.5, 0.5] and g[5] == 0.5 and int((g != 0).sum()) == 4
    del norm
    m, v = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    p = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    A.alch_adamw_step(A.AdamwList([p], [g], [m], [v]), 0.125)
    assert p[n - 4:].tolist() == [0.0, -0.125, -0.125, -0.125] and int((p != 0).sum()) == 4
    assert int((m != 0).sum()) == 4 and int((v != 0).sum()) == 4
