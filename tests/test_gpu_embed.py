"""alch_embed_forward and alch_embed_backward against their definitions.

The forward pass has one rounding: bits are compared.  A sum of the backward pass over n tokens has at most n - 1 additions
of 2^-24 each in whatever order, the product with the scale and the addition to the old value one each, the storage type half
a step: |error| <= half * |value| + 2^-24 * ((n + 1) * scale * sum |dX| + |old value|), per element, with
half = torch.finfo(type).eps / 2, and a second 2^-24 |value| for the rounding before it."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def randn(shape, dtype, seed, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std).to(DT[dtype])


def make_ids(kind, T, V, seed=0):
    r = np.random.default_rng(seed)
    if kind == "one":
        ids = np.full(T, V // 2)
    elif kind == "ascending":
        ids = np.arange(T) % V
    elif kind == "runs":      # two ids share most of the tokens
        ids = np.where(r.random(T) < 0.6, V - 1, np.where(r.random(T) < 0.5, 0, r.integers(0, V, T)))
    elif kind == "padding":   # no row at all
        ids = r.choice([-1, V, V + 7, -2 ** 31, 2 ** 31 - 1], T)
    else:                     # "mixed": some of them no row
        ids = np.where(r.random(T) < 0.2, r.choice([-1, V, -2 ** 31, 2 ** 31 - 1], T), r.integers(0, V, T))
    return ids.astype(np.int32)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,H,V,scale", [(1, 4096, 1000, 1.0), (1, 1, 1, 0.3), (487, 487, 97, 22.06), (33, 8, 50, 1.0), (5003, 256, 1000, -16.0),
                                         (70, 8200, 31, 64.0), (3, 20000, 5, 0.5), (999, 9, 20, 2.0), (5000, 3, 20, 1.0), (1000, 1029, 300, 1.0)])
def test_forward(T, H, V, scale, dtype):
    import paper_2503_01066_amd as A
    ids, W = make_ids("mixed", T, V), randn((V, H), dtype, 1)
    big = torch.full((T + 2, H), 7.0, dtype=DT[dtype], device="cuda")
    if H * big.element_size() % 16:
        X = A.alch_embed_forward(torch.from_numpy(ids).cuda(), W.cuda(), scale=scale)
    else:  # rows around the output stay as they were
        X = A.alch_embed_forward(torch.from_numpy(ids).cuda(), W.cuda(), scale=scale, X=big[1:T + 1])
        assert bool((big[0] == 7).all()) and bool((big[T + 1] == 7).all())
    ok = (ids >= 0) & (ids < V)
    ref = torch.zeros((T, H), dtype=DT[dtype])
    ref[ok] = (W[torch.from_numpy(ids[ok]).long()].float() * np.float32(scale)).to(DT[dtype])
    assert torch.equal(X.cpu(), ref)


def check_backward(ids, dX, V, scale, dW, old):
    """dW: device result; old: what it held (accumulate), or None."""
    T, H = dX.shape
    ok = (ids >= 0) & (ids < V)
    at, rows = torch.from_numpy(ids[ok]).long().cuda(), dX.cuda()[torch.from_numpy(np.flatnonzero(ok)).cuda()].double()
    n = torch.bincount(at, minlength=V).double()
    met, order = torch.nonzero(n)[:, 0], torch.argsort(at, stable=True)
    last = torch.cumsum(n[met].long(), 0) - 1

    def by_id(x):  # as differences of a running sum over the sorted tokens
        out, total = torch.zeros((V, H), dtype=torch.float64, device="cuda"), torch.cumsum(x[order], 0)[last]
        out[met] = total - torch.cat([torch.zeros_like(total[:1]), total[:-1]])
        return out

    ref, size = by_id(rows) * scale, by_id(rows.abs()) * abs(scale)
    before = torch.zeros_like(ref) if old is None else old.cuda().double()
    ref = ref + before
    half = torch.finfo(dX.dtype).eps / 2
    bound = (half + 2.0 ** -24) * ref.abs() + 2.0 ** -24 * ((n[:, None] + 1) * size + before.abs()) + 1e-44
    err = (dW.double() - ref).abs()
    assert bool(torch.isfinite(dW).all())
    assert bool((err <= bound).all()), float((err / bound).max())
    absent = n == 0
    assert torch.equal(dW[absent], torch.zeros_like(dW[absent]) if old is None else old.cuda()[absent])


CASES = [(1, 4096, 1000, "mixed"), (31, 256, 64, "mixed"), (32, 256, 64, "one"), (33, 487, 64, "one"), (64, 64, 3, "runs"), (65, 8, 1, "one"),
         (487, 4096, 5000, "mixed"), (487, 130, 128256, "ascending"), (1025, 72, 1023, "runs"), (1500, 40, 1024, "mixed"), (5003, 256, 1000, "runs"),
         (16384, 64, 128256, "runs"), (9000, 520, 7, "mixed"), (70001, 24, 40000, "one"), (200, 64, 9, "padding"), (300, 1, 17, "mixed"),
         (2049, 8200, 300, "runs"), (300, 8, 20, "runs"), (1024, 520, 40, "runs"), (777, 33, 2, "runs"), (16500, 2104, 500, "runs"),
         (16384, 1032, 90, "mixed"), (1025, 8, 20, "runs"), (1100, 264, 1, "one"), (1200, 64, 9, "padding"), (2000, 9, 31, "runs"), (90, 9, 31, "runs"),
         (3000, 515, 700, "mixed"), (8192, 100, 40, "runs"), (5000, 260, 999, "mixed"), (2500, 16, 2499, "ascending"), (3000, 70, 9, "padding"),
         (3500, 1032, 20000, "runs"), (2100, 40, 100000, "mixed"), (4096, 72, 128256, "one"), (1048581, 24, 3000, "runs"), (20000, 8, 3000000, "mixed"), (8193, 40, 30000, "mixed"), (4097, 16, 4097, "ascending")]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,H,V,kind", CASES)
def test_backward(T, H, V, kind, dtype):
    import paper_2503_01066_amd as A
    ids, dX = make_ids(kind, T, V, T), randn((T, H), dtype, T + 1, 0.01)
    bad = (ids < 0) | (ids >= V)
    dX[torch.from_numpy(bad)] = float("nan")  # rows without a token are not read
    dev_ids, dev = torch.from_numpy(ids).cuda(), dX.cuda()
    ws = torch.full((A.embed_backward_workspace_bytes(DT[dtype], V, H, T),), 0x7f, dtype=torch.uint8, device="cuda")
    whole = torch.full((V + 2, H), 3.0, dtype=DT[dtype], device="cuda")
    own = H * whole.element_size() % 16 == 0  # rows around the table stay as they were
    dW = whole[1:V + 1] if own else whole[:V].clone()
    A.alch_embed_backward(dev_ids, dev, V, scale=1.7, dW_embed=dW, workspace=ws)
    check_backward(ids, dX, V, np.float32(1.7).astype(np.float64), dW, None)
    old = randn((V, H), dtype, 5, 0.1)
    first = dW.clone()
    dW.copy_(old)
    A.alch_embed_backward(dev_ids, dev, V, scale=1.7, dW_embed=dW, accumulate=True, workspace=ws)
    check_backward(ids, dX, V, np.float32(1.7).astype(np.float64), dW, old)
    if own:
        assert bool((whole[0] == 3).all()) and bool((whole[V + 1] == 3).all())
    ws.fill_(0)  # what the workspace held makes no difference
    again = A.alch_embed_backward(dev_ids, dev, V, scale=1.7, workspace=ws)
    assert torch.equal(again, first)


@pytest.mark.parametrize("T,H,V", [(2100, 256, 800000), (5000, 256, 800000), (8000, 512, 410001), (3000, 2048, 100003), (5000, 5120, 40001), (2100, 6144, 40000)])
def test_few_tokens_of_a_large_table(T, H, V):
    """Most of the call writes zeros: rows of every width, and not a byte behind the table."""
    import paper_2503_01066_amd as A
    ids, dX = make_ids("mixed", T, V, 3), randn((T, H), "bf16", 4)
    ids[:700] = V - 1  # the last row, over many parts
    memory = torch.full((V + 1, H), 3.0, dtype=torch.bfloat16, device="cuda")
    dW = A.alch_embed_backward(torch.from_numpy(ids).cuda(), dX.cuda(), V, scale=0.5, dW_embed=memory[:V])
    check_backward(ids, dX, V, 0.5, dW, None)
    assert bool((memory[V] == 3).all())


def test_backward_without_tokens_writes_zeros():
    import paper_2503_01066_amd as A
    dW = torch.full((37, 24), 5.0, device="cuda")
    A.alch_embed_backward(torch.empty(0, dtype=torch.int32, device="cuda"), torch.empty(0, 24, device="cuda"), 37, dW_embed=dW)
    assert bool((dW == 0).all())
    dW.fill_(5.0)
    A.alch_embed_backward(torch.empty(0, dtype=torch.int32, device="cuda"), torch.empty(0, 24, device="cuda"), 37, dW_embed=dW, accumulate=True)
    assert bool((dW == 5).all())


@pytest.mark.parametrize("scale", [-2.0, float("inf"), float("nan")])
@pytest.mark.parametrize("T,V", [(40, 1000), (300, 50), (6000, 20000), (9000, 3000), (0, 9)])
def test_rows_without_a_token_are_zero_whatever_the_scale(T, V, scale):
    import paper_2503_01066_amd as A
    ids = (make_ids("mixed", T, V // 2, T) * 2) if T else np.empty(0, np.int32)  # (odd rows have no token)
    dev = torch.from_numpy(ids.astype(np.int32)).cuda()
    X = A.alch_embed_forward(dev, torch.ones(V, 72, device="cuda"), scale=scale)
    bad = torch.from_numpy((ids < 0) | (ids >= V)).cuda()
    assert X.shape == (T, 72) and bool((X[bad].view(torch.int32) == 0).all())
    dW = A.alch_embed_backward(dev, torch.ones(T, 72, device="cuda"), V, scale=scale, dW_embed=torch.full((V, 72), 5.0, device="cuda"))
    met = torch.zeros(V, dtype=torch.bool, device="cuda")
    met[dev[~bad].long()] = True
    assert bool((dW[~met].view(torch.int32) == 0).all()) and not bool((dW[met] == 0).any())


def test_infinities_and_nan_reach_their_own_row_alone():
    import paper_2503_01066_amd as A
    ids = np.array([3, 1, 3, 2, 1] * 20, np.int32)
    dX = torch.ones((100, 16))
    dX[0, 5], dX[1, 6], dX[3, 7], dX[8, 7] = float("inf"), float("nan"), float("inf"), -float("inf")
    dW = A.alch_embed_backward(torch.from_numpy(ids).cuda(), dX.cuda(), 5).cpu()
    assert dW[3, 5] == float("inf") and torch.isnan(dW[1, 6]) and torch.isnan(dW[2, 7])
    assert int((~torch.isfinite(dW)).sum()) == 3


def test_table_beyond_32_bit_offsets():
    import paper_2503_01066_amd as A
    V, H = 300000, 8192  # 2.46e9 elements
    W = torch.zeros((V, H), dtype=torch.bfloat16, device="cuda")
    W[V - 1].fill_(3.0)
    W[V - 2].fill_(2.0)
    ids = torch.tensor([V - 1, 0, V - 2, V - 1], dtype=torch.int32, device="cuda")
    X = A.alch_embed_forward(ids, W, scale=0.5)
    assert X[:, 0].tolist() == [1.5, 0.0, 1.0, 1.5] and bool((X == X[:, :1]).all())
    dW = A.alch_embed_backward(ids, X, V, dW_embed=W, accumulate=True)  # 3 + 3, 2 + 1
    assert dW[-1, 0] == 6 and dW[-2, 0] == 3 and bool((dW[-2:] == dW[-2:, :1]).all()) and bool((dW[:V - 2] == 0).all())
    dW = A.alch_embed_backward(ids, X, V, dW_embed=W)
    assert dW[-1, 0] == 3 and dW[-2, 0] == 1 and bool((dW[-2:] == dW[-2:, :1]).all()) and bool((dW[:V - 2] == 0).all())


def test_ids_of_31_bits():
    import paper_2503_01066_amd as A
    V, T = (1 << 30) + 77, 17000  # four digits
    r = np.random.default_rng(1)
    ids = np.concatenate([r.integers(0, V, T - 4000), np.full(2000, V - 1), r.choice([V, -1, 2 ** 31 - 1], 2000)]).astype(np.int32)
    r.shuffle(ids)
    dev = torch.from_numpy(ids).cuda()
    dX = torch.ones((T, 1), device="cuda")
    dW = torch.full((V, 1), 3.0, device="cuda")
    A.alch_embed_backward(dev, dX, V, dW_embed=dW)
    met, n = np.unique(ids[(ids >= 0) & (ids < V)], return_counts=True)
    at = torch.from_numpy(met).long().cuda()
    assert torch.equal(dW[at, 0], torch.from_numpy(n).float().cuda()) and int((dW != 0).sum()) == len(met)
    A.alch_embed_backward(dev, dX, V, dW_embed=dW, accumulate=True)
    assert torch.equal(dW[at, 0], torch.from_numpy(2 * n).float().cuda()) and int((dW != 0).sum()) == len(met)
    X = A.alch_embed_forward(dev, dW)
    ok = torch.from_numpy((ids >= 0) & (ids < V)).cuda()
    assert torch.equal(X[ok], dW[dev[ok].long()]) and bool((X[~ok] == 0).all())


def test_other_streams_and_two_calls_at_once():
    import paper_2503_01066_amd as A
    T, H, V = 3000, 512, 2000
    jobs = []
    for k in range(2):
        ids, dX = make_ids("runs", T, V, k), randn((T, H), "bf16", k)
        jobs.append((torch.from_numpy(ids).cuda(), dX.cuda(), torch.cuda.Stream(), torch.empty((V, H), dtype=torch.bfloat16, device="cuda")))
    alone = [A.alch_embed_backward(i, d, V) for i, d, _, _ in jobs]
    torch.cuda.synchronize()
    for rep in range(3):
        for ids, dX, s, dW in jobs:
            A.alch_embed_backward(ids, dX, V, dW_embed=dW, stream=s)
        torch.cuda.synchronize()
        for (_, _, _, dW), a in zip(jobs, alone):
            assert torch.equal(dW, a)


def test_gradient_against_differences():
    # f(W) = <R, X(W)> is linear in W: (f(W + h E) - f(W)) / h = <dW, E> up to rounding, for any direction E
    import paper_2503_01066_amd as A
    T, H, V, scale = 700, 48, 60, 3.0
    ids = make_ids("mixed", T, V)
    dev = torch.from_numpy(ids).cuda()
    W, R, E = (randn(s, "f32", k).cuda() for k, s in enumerate([(V, H), (T, H), (V, H)]))
    f = lambda w: (A.alch_embed_forward(dev, w, scale=scale).double() * R.double()).sum()
    dW = A.alch_embed_backward(dev, R, V, scale=scale)
    h = 0.5
    measured, formula = (f(W + h * E) - f(W)) / h, (dW.double() * E.double()).sum()
    # X and X(W + hE) are rounded twice (2^-24 of at most ~5 * 3 each), 33600 products with |R| ~ 1, over h: about 1e-4 of ~ 540
    assert abs(float(measured - formula)) <= 2.0 ** -23 * 2 / h * float((A.alch_embed_forward(dev, W.abs() + h * E.abs(), scale=scale) * R.abs()).double().sum()) + 1e-9


FORMS = ["plain", "fp32", "X", "no tokens", "whole scale", "64-bit ids", "ids of two dims", "spaced ids", "host ids", "host table", "half table", "table by columns",
         "X too short", "X of another type", "X by columns", "X on the host", "X off 16 bytes", "no table", "tensor scale", "another stream", "stream given"]


@pytest.mark.parametrize("form", FORMS)
def test_rows_marshalled_by_the_extension_and_in_python(monkeypatch, form):
    import paper_2503_01066_amd as A
    from paper_2503_01066_amd import binding
    assert binding._marshal is not None
    T, V, H = 5, 40, 64
    ids, W = torch.from_numpy(make_ids("mixed", T, V)).cuda(), randn((V, H), "bf16", 2).cuda()
    X, scale, stream, out = None, 0.75, None, []
    if form == "fp32": W = W.float()
    if form.startswith("X"): X = torch.full((T + 1, H), 9.0, dtype=W.dtype, device="cuda")[:T]
    if form == "no tokens": ids = ids[:0]
    if form == "whole scale": scale = 3
    if form == "64-bit ids": ids = ids.long()
    if form == "ids of two dims": ids = ids[None]
    if form == "spaced ids": ids = torch.stack([ids, ids], 1)[:, 0]
    if form == "host ids": ids = ids.cpu()
    if form == "host table": W = W.cpu()
    if form == "half table": W = W.half()
    if form == "table by columns": W = W.t().contiguous().t()
    if form == "X too short": X = X[:T - 1]
    if form == "X of another type": X = X.float()
    if form == "X by columns": X = X.t().contiguous().t()
    if form == "X on the host": X = X.cpu()
    if form == "X off 16 bytes": X = torch.zeros(T * H + 1, dtype=W.dtype, device="cuda")[1:].view(T, H)
    if form == "no table": W = None
    if form == "tensor scale": scale = torch.tensor(0.75)
    if form == "stream given": stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    for ext in (binding._marshal, None):
        monkeypatch.setattr(binding, "_marshal", ext)
        try:
            with torch.cuda.stream(torch.cuda.Stream() if form == "another stream" else None):
                got = A.alch_embed_forward(ids, W, scale=scale, X=X, stream=stream)
            torch.cuda.synchronize()
            out.append((got is X, got.dtype, got.tolist()))
        except Exception as e:  # noqa: BLE001 (compared below)
            out.append((type(e), str(e)))
    assert out[0] == out[1]
    fine = form in ("plain", "fp32", "X", "no tokens", "whole scale", "tensor scale", "another stream", "stream given")
    assert isinstance(out[0][0], bool) == fine
    if fine and form != "no tokens":
        ok = (ids >= 0) & (ids < V)
        want = torch.where(ok[:, None], (W[ids.long().clamp(0, V - 1)].float() * float(scale)).to(W.dtype), torch.zeros((), dtype=W.dtype, device="cuda"))
        assert out[0][2] == want.tolist()
