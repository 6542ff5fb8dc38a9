"""AdamW with moments in 8 bits at the ends of its scales: scale bytes whose power of two, times a beta, is no normal number of fp32 (or whose product with
a code is beyond it), betas down to 0.  Codes bit for bit, as everywhere."""
import numpy as np
import pytest
import torch

from test_gpu_adamw8 import DT, HYPER, reference, run

pytestmark = pytest.mark.gpu
N = 64 * 40 + 11


def states(kind):
    r = np.random.default_rng(5)
    m = r.integers(0, 256, N).astype(np.uint8)
    m[(m & 127) == 127] = 5
    v = r.integers(0, 256, N).astype(np.uint8)
    blocks = -(-N // 64)
    low, high = np.arange(blocks) % 8, np.arange(blocks) % 21
    ms = {"low": low, "high": 200 + high, "any": r.integers(0, 248, blocks)}[kind].astype(np.uint8)
    vs = {"low": low // 2, "high": 140 + high, "any": r.integers(0, 200, blocks)}[kind].astype(np.uint8)
    m[np.repeat(ms == 0, 64)[:N]] = 0
    v[np.repeat(vs == 0, 64)[:N]] = 0
    return (m, ms), (v, vs)


@pytest.mark.parametrize("dtype,master", [("f32", False), ("bf16", False), ("bf16", True), ("f32", True)])
@pytest.mark.parametrize("beta1,beta2", [(0.9, 0.999), (0.1, 0.9), (0.3, 0.05), (0.01, 0.5), (0.0, 0.0), (1e-6, 1e-6), (1e-30, 1e-36)])
@pytest.mark.parametrize("kind", ["low", "high", "any"])
@pytest.mark.parametrize("size", [0.0, 1e-30, 1.0])
def test_codes_at_the_ends(dtype, master, beta1, beta2, kind, size):
    import paper_2503_01066_amd as A
    g = torch.Generator(device="cuda").manual_seed(2)
    w = torch.randn(N, generator=g, device="cuda")
    grad = (torch.randn(N, generator=g, device="cuda") * size).to(DT[dtype])
    grad[::3] = 0
    before = [[w.to(DT[dtype]), grad, w + 1e-4 if master else None]]
    after = [[None if x is None else x.clone() for x in before[0]]]
    s = states(kind)
    hyper = dict(HYPER, beta1=beta1, beta2=beta2)
    ms, vs, firsts = run(A, after, [s], [0.1], step=3, **hyper)
    with np.errstate(all="ignore"):
        codes, nw, ew = reference(*before[0][:2], *s, before[0][2], float(np.float32(0.1)), 1.0, seed=7, first=0, step=3, **hyper)
    got = [t.cpu().numpy().reshape(-1) for t in ms[0] + vs[0]]
    for name, x, y in zip(("m", "m scale", "v", "v scale"), got, codes):
        assert np.array_equal(x, y), (name, np.nonzero(x != y)[0][:4], x[x != y][:4], y[x != y][:4])
    # weights where the step is a number that leaves some of the weight: |lr change| up to 1e6
    kept = after[0][2 if master else 0].double().cpu().numpy()
    fine = np.isfinite(nw) & np.isfinite(ew) & (np.abs(nw) < 1e6)
    bound = ew + (2.0 ** -8 * (np.abs(nw) + ew) if dtype == "bf16" and not master else 0)
    assert fine.any() and (np.abs(kept - nw) <= bound)[fine].all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("beta1", [0.1, 0.01])
def test_many_codes_of_the_smallest_scales(dtype, beta1):
    """2^(byte - 127) beta1 is below the normal numbers for bytes of 2 to 8, and would be a factor with fewer bits: a few codes in 100,000 then are others."""
    import paper_2503_01066_amd as A
    n = 1 << 20
    r = np.random.default_rng(8)
    m, v = (r.integers(8, 120, n).astype(np.uint8) for _ in range(2))
    s = (m, (2 + np.arange(n // 64) % 7).astype(np.uint8)), (v, np.full(n // 64, 90, np.uint8))
    before = [[torch.zeros(n, dtype=DT[dtype], device="cuda"), torch.zeros(n, dtype=DT[dtype], device="cuda"), None]]
    hyper = dict(HYPER, beta1=beta1)
    ms, vs, _ = run(A, [[x.clone() if x is not None else None for x in before[0]]], [s], [0.0], step=3, **hyper)
    codes, _, _ = reference(*before[0][:2], *s, None, 0.0, 1.0, seed=7, first=0, step=3, **hyper)
    for x, y in zip(ms[0] + vs[0], codes):
        assert np.array_equal(x.cpu().numpy(), y), np.count_nonzero(x.cpu().numpy() != y)
