"""Records in 8 bits against their definition, bit for bit: numpy makes the same roundings to fp32, one operation at a time.  What comes back is
half a step of its group off: |code * scale - x| <= scale * (1/2 + 127 * 3 * 2^-24) for the roundings of 127 / a, of the product and of the scale
itself on up to 127 steps, and then the storage type's own rounding of code * scale."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
TINY = np.float32(2.0 ** -100)


def quantised(x):
    """(codes, scales) of float32 rows."""
    rows, width = x.shape
    groups = -(-width // 64)
    p = np.zeros((rows, groups * 64), np.float32)
    p[:, :width] = x
    p = p.reshape(rows, groups, 64)
    with np.errstate(all="ignore"):
        a = np.abs(p).max(2)
        fine, some = np.isfinite(a), a >= TINY
        r = np.where(fine & some, np.float32(127) / a, np.float32(0)).astype(np.float32)
        codes = np.where(fine[:, :, None], np.rint(np.where(fine[:, :, None], p, 0) * r[:, :, None]), 0)
        scales = np.where(fine, np.where(some, a / np.float32(127), np.float32(0)), np.float32(np.nan)).astype(np.float32)
    return codes.reshape(rows, groups * 64)[:, :width].astype(np.int8), scales


def values(rows, width, dtype, seed, pad=0):
    """Rows of a wider buffer, pad elements before and behind them; single groups with what is hard to hold."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    wide = torch.randn((rows, width + 2 * pad), generator=g, device="cuda")
    wide *= torch.exp(torch.randn((rows, 1), generator=g, device="cuda") * 3)
    x = wide[:, pad:pad + width]
    for i, special in enumerate((0.0, np.inf, -np.inf, np.nan, 1e-38, 1e-42, 3e38, -0.0)):
        r = 3 * i + 1
        if r < rows:
            if i in (0, 4, 5, 7):
                x[r, :min(width, 70)] = special
            else:
                x[r, (5 * i) % width] = special
    t = wide.to(DT[dtype])
    return t[:, pad:pad + width]


def host(t):
    return t.detach().float().cpu().numpy()


def same(a, b):
    return np.array_equal(a.view(np.uint8) if a.dtype == np.int8 else a, b.view(np.uint8) if b.dtype == np.int8 else b, equal_nan=a.dtype != np.int8)


def check(A, mask, streams, capacity=None, cu=None, **kw):
    T = len(mask)
    b = A.Batch(np.array([0, T], np.int32) if cu is None else cu)
    kept = np.nonzero(mask)[0]
    cap = T if capacity is None else capacity
    dsts = [(torch.full((cap, s.shape[1]), 77, dtype=torch.int8, device="cuda"), torch.full((cap, -(-s.shape[1] // 64)), 7.5, device="cuda")) for s in streams]
    index, cu_kept, status, out = A.alch_capture_pack_q8(b, torch.from_numpy(mask).cuda(), streams, capacity=cap, dsts=dsts, **kw)
    torch.cuda.synchronize()
    n = min(len(kept), cap)
    assert status.tolist() == [len(kept), int(len(kept) > cap)] and index[:n].tolist() == kept[:n].tolist()
    assert cu_kept.tolist() == [int((kept < c).sum()) for c in b.cu_host]
    for k, (s, (codes, scales)) in enumerate(zip(streams, out)):
        want = quantised(host(s)[kept[:n]])
        assert same(codes[:n].cpu().numpy(), want[0]) and same(scales[:n].cpu().numpy(), want[1]), k
        assert bool((codes[n:] == 77).all()) and bool((scales[n:] == 7.5).all()), k
    return index, status, out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("width", [1, 7, 8, 63, 64, 65, 72, 128, 487, 2056, 4096])
def test_pack_widths(dtype, width):
    import paper_2503_01066_amd as A
    T = 57
    mask = (np.arange(T) % 3 != 2).astype(np.uint8) * 5
    streams = [values(T, width, dtype, 1), values(T, width, dtype, 2, pad=8), values(T, width, dtype, 3, pad=1)]
    check(A, mask, streams)


@pytest.mark.parametrize("T,keep", [(1, 1.0), (1, 0.0), (16, 0.0), (300, 1.0), (4095, 0.5), (4096, 0.02), (4097, 0.3), (8192, 0.02), (8192, 1.0), (8193, 0.1), (9000, 0.9), (270001, 0.01)])
def test_pack_lengths_and_masks(T, keep):
    import paper_2503_01066_amd as A
    r = np.random.default_rng(T)
    mask = (r.random(T) < keep).astype(np.uint8)
    streams = [values(T, w, d, w) for w, d in ((256, "bf16"), (72, "f32"), (33, "bf16"), (12, "f32"))]
    inner = np.sort(r.integers(0, T + 1, 6))
    cu = np.concatenate([[0], inner, [T]]).astype(np.int32)
    check(A, mask, streams, cu=cu)
    if mask.sum() > 1:
        check(A, mask, streams, cu=cu, capacity=int(mask.sum()) // 2)
        check(A, mask, streams, cu=cu, capacity=int(mask.sum()))


def test_pack_of_nothing():
    import paper_2503_01066_amd as A
    check(A, np.zeros(0, np.uint8), [torch.zeros((0, 64), dtype=torch.bfloat16, device="cuda")], cu=np.array([0, 0], np.int32))
    check(A, np.ones(5, np.uint8), [])
    check(A, np.ones(5, np.uint8), [values(5, 64, "bf16", 1)], capacity=0)
    assert A.alch_record_expand([]) == []


def test_many_streams_and_the_gather():
    import paper_2503_01066_amd as A
    T = 700
    mask = (np.random.default_rng(0).random(T) < 0.4).astype(np.uint8)
    fused = values(T, 64 * 20 + 40, "bf16", 9)
    streams = [fused[:, 64 * k:64 * k + w] for k, w in enumerate([64, 8, 40, 64, 63, 1] * 3 + [104, 64])]
    index, status, out = check(A, mask, streams)
    n = int(mask.sum())
    b = A.Batch(np.array([0, T], np.int32))
    again = A.alch_capture_gather_q8(b, streams, index, status, capacity=T)
    assert all(torch.equal(x[:n], y[:n]) for p, q in zip(out, again) for x, y in zip(p, q))
    few = A.alch_capture_gather_q8(b, streams[:2], index, status, dsts=[(p[0][:10].clone(), p[1][:10].clone()) for p in out[:2]])
    assert all(torch.equal(x, y[:10]) for p, q in zip(few, out) for x, y in zip(p, q))
    whole = A.alch_capture_gather_q8(b, streams)
    for s, (codes, scales) in zip(streams, whole):
        want = quantised(host(s))
        assert same(codes.cpu().numpy(), want[0]) and same(scales.cpu().numpy(), want[1])
    # an index of a pack in full width serves as well
    kept, _, st, _ = A.alch_capture_pack(b, torch.from_numpy(mask).cuda(), [])
    other = A.alch_capture_gather_q8(b, streams[:3], kept, st)
    assert all(torch.equal(x[:n], y[:n]) for p, q in zip(out, other) for x, y in zip(p, q))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("width", [1, 8, 63, 64, 72, 487, 4096])
@pytest.mark.parametrize("how", ["all", "rows", "slices"])
def test_expand(dtype, width, how):
    import paper_2503_01066_amd as A
    held, widths = 90, [width, 64, max(width // 3, 1)]
    src = [values(held, w, "f32", w) for w in widths]
    pairs = A.alch_capture_gather_q8(A.Batch(np.array([0, held], np.int32)), src)
    if how == "all":
        at, rows, outs = np.arange(held), None, None
    else:
        at = np.array([3, 3, 0, 89, -1, 90, 2 ** 31 - 1, -2 ** 31, 17, 88, 3] * 9, np.int32)
        rows = torch.from_numpy(at.astype(np.int32)).cuda()
        outs = None
    n = len(at)
    if how == "slices":
        pad = 8 if width % 8 == 0 else 1
        wide = torch.full((n, sum(widths) + 4 * pad), 9.0, dtype=DT[dtype], device="cuda")
        cuts, outs = [], []
        c = pad
        for w in widths:
            outs.append(wide[:, c:c + w])
            cuts.append((c, w))
            c += w + pad
    got = A.alch_record_expand(pairs, outs=outs, rows=rows, dtype=DT[dtype])
    torch.cuda.synchronize()
    for k, ((codes, scales), o) in enumerate(zip(pairs, got)):
        v = codes.float().cpu() * scales.cpu().repeat_interleave(64, 1)[:, :widths[k]]
        good = torch.from_numpy((at >= 0) & (at < held))
        want = torch.zeros((n, widths[k]))
        want[good] = v[torch.from_numpy(at)[good].long()]
        assert torch.equal(torch.nan_to_num(o.cpu().float(), nan=1e9), torch.nan_to_num(want.to(DT[dtype]).float(), nan=1e9)), k
        if how == "all":  # and near what was captured
            x = src[k].double().cpu()
            s = scales.double().cpu().repeat_interleave(64, 1)[:, :widths[k]]
            fine = torch.isfinite(s) & (s > 0)
            off = (o.double().cpu() - x).abs()
            bound = s * (0.5 + 381 * 2.0 ** -24) + torch.finfo(DT[dtype]).eps / 2 * (x.abs() + s)
            assert bool((off <= bound)[fine].all())
    if how == "slices":
        outside = torch.ones(wide.shape[1], dtype=torch.bool)
        for c, w in cuts:
            outside[c:c + w] = False
        assert bool((wide[:, outside.cuda()] == 9.0).all())


def test_largest_of_a_group_comes_back():
    import paper_2503_01066_amd as A
    x = values(500, 640, "bf16", 4)[25:]  # (without the rows of infinities)
    back, = A.alch_record_expand(A.alch_capture_gather_q8(A.Batch(np.array([0, len(x)], np.int32)), [x.contiguous()]))
    g, h = x.float().view(-1, 64), back.float().view(-1, 64)
    at = g.abs().argmax(1, keepdim=True)
    assert torch.equal(g.gather(1, at), h.gather(1, at))  # (127 * fl(a / 127) is within 2^-24 of a, which bf16 rounds away)


def test_first_rows_and_refusals():
    import paper_2503_01066_amd as A
    b = A.Batch(np.array([0, 20], np.int32))
    x = values(20, 128, "bf16", 1)
    (codes, scales), = pairs = A.alch_capture_gather_q8(b, [x])
    assert torch.equal(A.alch_record_expand(pairs, n_rows=7)[0].nan_to_num(), A.alch_record_expand(pairs)[0][:7].nan_to_num())
    for call in (lambda: A.alch_record_expand([(codes, scales[:, :1])]), lambda: A.alch_record_expand([(codes.int(), scales)]),
                 lambda: A.alch_record_expand(pairs, outs=[torch.empty(19, 128, device="cuda")]), lambda: A.alch_record_expand(pairs + [(codes[:5], scales[:5])]),
                 lambda: A.alch_record_expand(pairs, rows=torch.zeros(3, dtype=torch.int64, device="cuda")), lambda: A.alch_capture_gather_q8(b, [x[:, ::2]]),
                 lambda: A.alch_capture_gather_q8(b, [x[:19]]), lambda: A.alch_capture_gather_q8(b, [x.cpu()]),
                 lambda: A.alch_capture_pack_q8(b, torch.ones(19, dtype=torch.uint8, device="cuda"), [x]),
                 lambda: A.alch_capture_pack_q8(b, torch.ones(20, dtype=torch.uint8, device="cuda"), [x], capacity=30, dsts=pairs)):
        with pytest.raises(ValueError):
            call()
    out = torch.empty((20, 128), dtype=torch.bfloat16, device="cuda")
    for call in (lambda: A.alch_record_expand(pairs, n_rows=21), lambda: A.alch_record_expand(pairs * 2, outs=[out] * 2),
                 lambda: A.alch_record_expand(pairs, outs=[codes.view(torch.bfloat16).view(10, 128)], n_rows=10)):
        with pytest.raises(A.AlchError):
            call()
    with pytest.raises(TypeError):
        A.alch_capture_gather_q8(b, [x.half()])


@pytest.mark.parametrize("form", ["lists", "tuples", "slices", "many", "columns apart", "host", "half", "rows", "codes", "scales", "no pair", "unequal", "none"])
def test_entries_by_the_extension_and_in_python(monkeypatch, form):
    """The same results, and the same errors for what either refuses."""
    import paper_2503_01066_amd as A
    from paper_2503_01066_amd import binding
    assert binding._marshal is not None
    T = 40
    wide = values(T, 400, "bf16", 5)
    streams = [wide[:, :64], wide[:, 64:163], wide[:, 168:].float()]
    dsts = [[torch.zeros((T, s.shape[1]), dtype=torch.int8, device="cuda"), torch.zeros((T, -(-s.shape[1] // 64)), device="cuda")] for s in streams]
    if form == "tuples": streams, dsts = tuple(streams), tuple(tuple(d) for d in dsts)
    if form == "many": streams, dsts = streams * 30, [[c.clone(), s.clone()] for c, s in dsts * 30]
    if form == "columns apart": streams[1] = wide[:, 1:199:2]
    if form == "host": streams[2] = streams[2].cpu()
    if form == "half": streams[0] = streams[0].half()
    if form == "rows": streams[1] = streams[1][:39]
    if form == "codes": dsts[1][0] = dsts[1][0].int()
    if form == "scales": dsts[1][1] = dsts[1][1][:, :1]
    if form == "no pair": dsts = dsts[:2]
    if form == "unequal": dsts[0] = [t[:30] for t in dsts[0]]
    if form == "none": streams, dsts = [], []
    mask = (torch.arange(T, device="cuda") % 3 == 0).to(torch.uint8)
    out = []
    for ext in (binding._marshal, None):
        monkeypatch.setattr(binding, "_marshal", ext)
        for pair in dsts:
            for t in pair:
                t.zero_()
        try:
            index, cu, status, d = A.alch_capture_pack_q8(A.Batch(np.array([0, 13, T], np.int32)), mask, streams, dsts=dsts)
            back = A.alch_record_expand(d) if form != "unequal" else []
            out.append([t.tolist() for t in (index[:14], cu, status)] + [t.nan_to_num().tolist() for p in d for t in p] + [t.float().nan_to_num().tolist() for t in back])
        except Exception as e:  # noqa: BLE001 (compared below)
            out.append((type(e), str(e)))
    assert out[0] == out[1]
    assert isinstance(out[0], tuple) == (form in ("columns apart", "host", "half", "rows", "codes", "scales", "no pair"))


def test_calls_on_another_stream_and_captured():
    import paper_2503_01066_amd as A
    T = 3000
    b = A.Batch(np.array([0, 1000, 3000], np.int32))
    masks = [(np.random.default_rng(k).random(T) < 0.3).astype(np.uint8) for k in range(3)]
    mask = torch.zeros(T, dtype=torch.uint8, device="cuda")
    x = [torch.zeros((T, w), dtype=torch.bfloat16, device="cuda") for w in (256, 72)]
    inputs = [[values(T, w, "bf16", 10 * k + w)[:] for w in (256, 72)] for k in range(3)]
    ws = torch.empty(A.lib().alch_capture_pack_workspace_bytes(T), dtype=torch.uint8, device="cuda")
    rows = torch.from_numpy(np.arange(T, dtype=np.int32)).cuda()

    def call(stream=None):
        out = A.alch_capture_pack_q8(b, mask, x, workspace=ws, stream=stream)
        return out[:3], out[3], A.alch_record_expand(out[3], rows=rows, stream=stream)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    call(s)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = call()
    for k in (0, 1, 2, 1):
        mask.copy_(torch.from_numpy(masks[k]))
        for a, v in zip(x, inputs[k]):
            a.copy_(v)
        torch.cuda.synchronize()
        want = call()
        other = call(s)
        graph.replay()
        torch.cuda.synchronize()
        n = int(masks[k].sum())
        for got in (captured, other):
            assert torch.equal(got[0][0][:n], want[0][0][:n]) and torch.equal(got[0][1], want[0][1]) and torch.equal(got[0][2], want[0][2])
            for p, q in zip(got[1], want[1]):
                assert torch.equal(p[0][:n], q[0][:n]) and torch.equal(p[1][:n].nan_to_num(), q[1][:n].nan_to_num())
            assert all(torch.equal(p[:n].nan_to_num(), q[:n].nan_to_num()) for p, q in zip(got[2], want[2]))


def test_offsets_beyond_32_bits():
    import paper_2503_01066_amd as A
    rows, width = 270000, 8192  # 2.2e9 codes, 4.4 GB of bf16
    x = torch.zeros((rows, width), dtype=torch.bfloat16, device="cuda")
    x[-1] = torch.arange(width, device="cuda").bfloat16()
    x[-2, 5] = -3.0
    (codes, scales), = pairs = A.alch_capture_gather_q8(A.Batch(np.array([0, rows], np.int32)), [x])
    want = quantised(host(x[-2:]))
    assert same(codes[-2:].cpu().numpy(), want[0]) and same(scales[-2:].cpu().numpy(), want[1]) and int((codes != 0).sum()) == int((want[0] != 0).sum())
    del x
    back, = A.alch_record_expand(pairs)
    one, = A.alch_record_expand(pairs, rows=torch.tensor([rows - 1, 0], dtype=torch.int32, device="cuda"))
    assert torch.equal(back[-1], one[0]) and int((back != 0).sum()) == int((want[0] != 0).sum()) and back[-2, 5] == -3.0


@pytest.mark.parametrize("width", [40, 2000])
def test_an_index_that_is_no_token_leaves_its_row(width):
    import paper_2503_01066_amd as A
    T = 9
    x = values(T, width, "bf16", 4)
    index = torch.tensor([-1, 3, T, 2 ** 31 - 1, 8, -2 ** 31, 0], dtype=torch.int32, device="cuda")
    status = torch.tensor([7, 0], dtype=torch.int32, device="cuda")
    dsts = [(torch.full((7, width), 77, dtype=torch.int8, device="cuda"), torch.full((7, -(-width // 64)), 7.5, device="cuda"))]
    (codes, scales), = A.alch_capture_gather_q8(A.Batch(np.array([0, T], np.int32)), [x], kept_index=index, status=status, dsts=dsts)
    want, wscales = quantised(host(x)[[3, 8, 0]])
    assert same(codes.cpu().numpy()[[1, 4, 6]], want) and same(scales.cpu().numpy()[[1, 4, 6]], wscales)
    rest = [0, 2, 3, 5]
    assert bool((codes[rest] == 77).all()) and bool((scales[rest] == 7.5).all())
    # the index of a call without room: one element that nothing wrote, and as many kept tokens as there are
    mask = torch.ones(T, dtype=torch.uint8, device="cuda")
    index, _, status, _ = A.alch_capture_pack_q8(A.Batch(np.array([0, T], np.int32)), mask, [x], capacity=0)
    assert status.tolist() == [T, 1]
    index.fill_(-5)
    dsts = [(torch.full((1, width), 77, dtype=torch.int8, device="cuda"), torch.full((1, -(-width // 64)), 7.5, device="cuda"))]
    (codes, scales), = A.alch_capture_gather_q8(A.Batch(np.array([0, T], np.int32)), [x], kept_index=index, status=status, dsts=dsts)
    assert bool((codes == 77).all()) and bool((scales == 7.5).all())
