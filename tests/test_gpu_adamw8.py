"""AdamW with moments in 8 bits against its definition: the codes and scales bit for bit (numpy makes the same fp32 operations one at a time,
the random bits are whole numbers), the weights with the tolerances of the update with fp32 moments, whose roundings they have from there on."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
U = 2.0 ** -24
HYPER = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8)
SIZES = [0, 1, 3, 4, 63, 64, 65, 255, 1000, 1023, 1024, 1025, 0, 4097, 100003]
M32 = np.uint64(0xffffffff)


def mix(x):
    x = np.asarray(x, dtype=np.uint64)
    x = x ^ (x >> np.uint64(16))
    x = (x * np.uint64(0x6A09E667)) & M32
    x = x ^ (x >> np.uint64(15))
    x = (x * np.uint64(0xBB67AE85)) & M32
    return x ^ (x >> np.uint64(16))


def random_bits(seed, step, first, n):
    i = np.uint64(first) + np.arange(n, dtype=np.uint64)
    return mix(((i & M32) + mix(mix(np.uint64(seed) ^ mix(np.uint64(step))) ^ (i >> np.uint64(32)))) & M32)


def blocks(x):
    p = np.zeros(-(-len(x) // 64) * 64, x.dtype)
    p[:len(x)] = x
    return p.reshape(-1, 64)


def scale_values(s):
    return np.where(s == 255, np.float32(np.nan), (s.astype(np.uint32) << 23).view(np.float32)).astype(np.float32)


def decode(codes, scales, which):
    c = codes.astype(np.int64)
    if which == "m":
        e, f = (c >> 3) & 15, c & 7
        y = np.where(e > 0, (1 + f / 8) * 2.0 ** (e - 7), f * 2.0 ** -9) * np.where(c >> 7, -1, 1)
        y = np.where((c & 127) == 127, np.nan, y)
    else:
        e, f = c >> 3, c & 7
        y = np.where(e > 0, (1 + f / 8) * 2.0 ** (e - 15), f * 2.0 ** -17)
    return (y.astype(np.float32) * np.repeat(scale_values(scales), 64)[:len(c)]).astype(np.float32)


def encode(x, bits16, which):
    """float32 values -> (codes, scales)"""
    n, above, lowest = len(x), (7 if which == "m" else 15), (-6 if which == "m" else -14)
    b = blocks(x)
    with np.errstate(all="ignore"):
        exponent = (np.abs(b).max(1).view(np.uint32) >> 23).astype(np.int64)
        s = np.where(exponent == 255, 255, np.maximum(exponent - above, 1))
        y = (b * ((254 - np.minimum(s, 253)).astype(np.uint32) << 23).view(np.float32)[:, None]).reshape(-1)[:n]
        sign, y = np.signbit(y), np.abs(y)
        small = y < 2.0 ** lowest
        t = np.where(small, y + np.float32(2.0 ** lowest), y).astype(np.float32).view(np.uint32).astype(np.int64)
    code = ((t + (bits16.astype(np.int64) << 4)) >> 20) - np.where(small, (127 + lowest) * 8, (126 + lowest) * 8)
    if which == "m":
        code |= sign.astype(np.int64) << 7
    else:
        code = np.where((x > 0) & (code == 0), 1, code)
    code = np.where(np.repeat(s == 255, 64)[:n], 127 if which == "m" else 255, code)
    return code.astype(np.uint8), s.astype(np.uint8)


def reference(p, g, m, v, w, decay, f, lr, beta1, beta2, eps, step, seed, first):
    """(codes and scales of m and v, weights in 64 bits, their bound)"""
    f32 = np.float32
    g, old = g.float().cpu().numpy().reshape(-1), (p if w is None else w).double().cpu().numpy().reshape(-1)
    mo, vo = decode(*m, "m"), decode(*v, "v")
    with np.errstate(all="ignore"):
        x = g * f32(f)
        nm = mo * f32(beta1) + x * f32(1 - beta1)
        nv = vo * f32(beta2) + (x * x) * f32(1 - beta2)
        bits = random_bits(seed, step, first, len(g))
        codes = encode(nm, bits & np.uint64(0xffff), "m") + encode(nv, bits >> np.uint64(16), "v")
        c1, den = 1 / (1 - beta1 ** step), np.sqrt(nv.astype(np.float64) / (1 - beta2 ** step)) + eps
        change = nm.astype(np.float64) * c1 / den
        nw = old - lr * (change + decay * old)
    ew = lr * (16 * U * np.abs(change) + 6 * U * np.abs(decay * old)) + U * (np.abs(nw) + lr * np.abs(change + decay * old)) + 1e-44
    return codes, nw, ew


def state(n, seed, scale):
    """Moments as a run leaves them: any codes, scales of ordinary size."""
    r = np.random.default_rng(seed)
    m = r.integers(0, 256, n).astype(np.uint8)
    m[(m & 127) == 127] = 5
    v = r.integers(1, 256, n).astype(np.uint8)
    s = lambda lo: (r.integers(lo, lo + 6, -(-n // 64))).astype(np.uint8)
    return (m, s(127 - 7 + scale)), (v, s(127 - 15 + 2 * scale))


def run(A, tensors, states, decay, first=None, grad_factor=None, seed=7, schedule=None, **hyper):
    dev = lambda pair, p: (torch.from_numpy(pair[0]).cuda().view(p.shape), torch.from_numpy(pair[1]).cuda())
    ms, vs = [dev(s[0], t[0]) for s, t in zip(states, tensors)], [dev(s[1], t[0]) for s, t in zip(states, tensors)]
    masters = [t[2] for t in tensors]
    l = A.Adamw8List([t[0] for t in tensors], [t[1] for t in tensors], ms, vs, masters=None if masters[0] is None else masters, weight_decay=decay, first=first)
    A.alch_adamw8_step(l, seed=seed, grad_factor=grad_factor, schedule=schedule, **hyper)
    torch.cuda.synchronize()
    return ms, vs, [r.first for r in l.host][:len(tensors)]


def make(sizes, dtype, master, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = []
    for n in sizes:
        w = torch.randn(n, generator=g, device="cuda")
        grad = (torch.randn(n, generator=g, device="cuda") * torch.exp(2 * torch.randn(n, generator=g, device="cuda")) * 0.01).to(DT[dtype])
        if n > 200:
            grad[100:200] = 0
        out.append([w.to(DT[dtype]), grad, w + 1e-4 if master else None])
    return out


def check(before, states, after, ms, vs, firsts, decay, f, seed, **hyper):
    for i, (b, s, a) in enumerate(zip(before, states, after)):
        codes, nw, ew = reference(*b[:2], *s, b[2], float(np.float32(decay[i])), 1.0 if f is None else f, seed=seed, first=firsts[i], **hyper)
        got = [t.cpu().numpy().reshape(-1) for t in ms[i] + vs[i]]
        for name, x, y in zip(("m", "m scale", "v", "v scale"), got, codes):
            assert np.array_equal(x, y), (i, name, np.nonzero(x != y)[0][:4], x[x != y][:4], y[x != y][:4])
        w = a[0] if b[2] is None else a[2]
        err = np.abs(w.double().cpu().numpy() - nw)
        bound = ew + (2.0 ** -8 * (np.abs(nw) + ew) if w.dtype == torch.bfloat16 else 0)
        assert bool((err <= bound).all()), (i, float((err / bound).max()))
        if b[2] is not None:
            assert torch.equal(a[0], a[2].to(a[0].dtype))


@pytest.mark.parametrize("dtype,master", [("f32", False), ("bf16", False), ("bf16", True), ("f32", True)])
@pytest.mark.parametrize("step,factor", [(1, None), (7, 0.25), (100000, 1.0)])
def test_step(dtype, master, step, factor):
    import paper_2503_01066_amd as A
    before, decay = make(SIZES, dtype, master, 1), [0.1 if i % 2 else 0.0 for i in range(len(SIZES))]
    states = [state(n, i, -7) for i, n in enumerate(SIZES)]
    if step == 1:
        states = [tuple((np.zeros(n, np.uint8), np.zeros(-(-n // 64), np.uint8)) for _ in range(2)) for n in SIZES]
    after = [[None if x is None else x.clone() for x in t] for t in before]
    fac = None if factor is None else torch.full((1,), factor, device="cuda")
    ms, vs, firsts = run(A, after, states, decay, grad_factor=fac, step=step, seed=step * 977, **HYPER)
    check(before, states, after, ms, vs, firsts, decay, factor, seed=step * 977, step=step, **HYPER)


def test_numbers_beyond_32_bits_and_tensors_in_pieces():
    """The same elements in one tensor, in pieces of whole blocks and in another order give the same bits."""
    import paper_2503_01066_amd as A
    n, at = 64 * 70 + 13, (1 << 33) - 64 * 20
    whole = make([n], "bf16", True, 3)
    s = state(n, 5, -7)
    a = [[x.clone() for x in whole[0]]]
    ms, vs, firsts = run(A, a, [s], [0.1], first=[at], step=9, **HYPER)
    check(whole, [s], a, ms, vs, firsts, [0.1], None, seed=7, step=9, **HYPER)
    cuts = [(64 * 33, n), (0, 64), (64, 64 * 33)]
    pieces = [[x[i:j].clone() for x in whole[0]] for i, j in cuts]
    parts = [tuple((c[i:j], sc[i // 64:-(-j // 64)]) for c, sc in s) for i, j in cuts]
    ms2, vs2, _ = run(A, pieces, parts, [0.1] * 3, first=[at + i for i, j in cuts], step=9, **HYPER)
    for (i, j), t, m, v in zip(cuts, pieces, ms2, vs2):
        assert torch.equal(t[0], a[0][0][i:j]) and torch.equal(t[2], a[0][2][i:j])
        assert torch.equal(m[0], ms[0][0][i:j]) and torch.equal(v[0], vs[0][0][i:j]) and torch.equal(m[1], ms[0][1][i // 64:-(-j // 64)])


@pytest.mark.parametrize("n", [63, 64, 65, 300, 4096])
def test_many_tensors(n):
    import paper_2503_01066_amd as A
    sizes = np.random.default_rng(n).integers(0, 200, n).tolist()
    before = make(sizes, "bf16", False, n)
    states = [state(k, i, -7) for i, k in enumerate(sizes)]
    after = [[x.clone() if x is not None else None for x in t] for t in before]
    ms, vs, firsts = run(A, after, states, [0.1] * n, step=3, **HYPER)
    few = list(range(0, n, max(n // 60, 1)))
    pick = lambda l: [l[i] for i in few]
    check(pick(before), pick(states), pick(after), pick(ms), pick(vs), pick(firsts), [0.1] * n, None, seed=7, step=3, **HYPER)


def test_scales_of_any_alignment_and_what_lies_between():
    import paper_2503_01066_amd as A
    sizes, flat = [100, 64, 1, 1500], 4096
    g = torch.Generator(device="cuda").manual_seed(1)
    p, grad = (torch.randn(flat, generator=g, device="cuda").bfloat16() for _ in range(2))
    codes = [torch.randint(1, 120, (flat,), generator=g, device="cuda").to(torch.uint8) for _ in range(2)]
    scales = [torch.full((80,), k, dtype=torch.uint8, device="cuda") for k in (115, 100)]
    at, bl = [0, 112, 192, 208], [1, 4, 6, 8]  # (elements between the tensors and scale bytes between their scales)
    cut = lambda x: [x[a:a + n] for a, n in zip(at, sizes)]
    sc = lambda x: [x[b:b + -(-n // 64)] for b, n in zip(bl, sizes)]
    old = [x.clone() for x in [p] + codes + scales]
    A.alch_adamw8_step(A.Adamw8List(cut(p), cut(grad), list(zip(cut(codes[0]), sc(scales[0]))), list(zip(cut(codes[1]), sc(scales[1])))), 0.1, step=4)
    inside, blocks_in = torch.zeros(flat, dtype=torch.bool, device="cuda"), torch.zeros(80, dtype=torch.bool, device="cuda")
    for a, b, n in zip(at, bl, sizes):
        inside[a:a + n] = True
        blocks_in[b:b + -(-n // 64)] = True
    for x, y in zip([p] + codes, old):
        assert torch.equal(x[~inside], y[~inside])
    assert not torch.equal(p[inside], old[0][inside])
    for x, y in zip(scales, old[3:]):
        assert torch.equal(x[~blocks_in], y[~blocks_in])


def test_values_that_are_no_numbers_and_extremes():
    import paper_2503_01066_amd as A
    n = 64 * 12
    grad = torch.zeros(n, device="cuda")
    for b, x in enumerate((math.nan, math.inf, -math.inf, 1e-45, 1e-38, 1e19, 1.9e19, 3e38, 1e-30, 1.0, -1.0, 0.0)):
        grad[64 * b + b] = x
        grad[64 * b + 40] = 1e-5
    before = [[torch.ones(n, device="cuda"), grad, None]]
    zeros = lambda: (np.zeros(n, np.uint8), np.zeros(n // 64, np.uint8))
    after = [[x.clone() if x is not None else None for x in before[0]]]
    ms, vs, firsts = run(A, after, [(zeros(), zeros())], [0.0], step=1, **HYPER)
    (mc, msc), (vc, vsc), nw, _ = (lambda c, w, e: ((c[0], c[1]), (c[2], c[3]), w, e))(*reference(*before[0][:2], zeros(), zeros(), None, 0.0, 1.0, seed=7, first=0, step=1, **HYPER))
    for x, y in zip(ms[0] + vs[0], (mc, msc, vc, vsc)):
        assert np.array_equal(x.cpu().numpy(), y)
    assert (msc[:3] == 255).all() and (vsc[[0, 1, 2, 6, 7]] == 255).all() and msc[5] != 255
    p = after[0][0].view(-1, 64)
    assert bool(torch.isfinite(p[3:6]).all()) and bool((p[11, :40] == 1).all())
    # such a block stays what it is, its neighbours do not
    again = [[x.clone() if x is not None else None for x in after[0]]]
    again[0][1] = torch.full((n,), 0.01, device="cuda")
    st = lambda pair: tuple(t.cpu().numpy() for t in pair)
    ms2, vs2, _ = run(A, again, [(st(ms[0]), st(vs[0]))], [0.0], step=2, **HYPER)
    assert ms2[0][1].cpu().numpy()[:3].tolist() == [255] * 3 and bool(torch.isnan(again[0][0].view(-1, 64)[:3]).all())
    assert bool(torch.isfinite(again[0][0].view(-1, 64)[8:]).all())


def test_second_moments_near_the_smallest_numbers():
    """Their roots are divided by as they are, without eps too."""
    import paper_2503_01066_amd as A
    n = 64 * 9 + 5
    r = np.random.default_rng(3)
    grad = torch.from_numpy((10.0 ** r.uniform(-22, -13, n) * r.choice([-1, 1], n)).astype(np.float32)).cuda()
    grad[:64] = torch.from_numpy((10.0 ** r.uniform(-19.5, -18.5, 64)).astype(np.float32)).cuda()
    grad[64] = 1.0  # (a block of usual size with tiny ones in it)
    grad = torch.where(grad.abs() < 3e-21, torch.zeros_like(grad), grad)  # (whose squares, times 1 - beta2, would be no numbers but 0)
    grad[(grad.double().square() * 0.001).float() == 0] = 0
    before = [[torch.ones(n, device="cuda"), grad, None]]
    zeros = (np.zeros(n, np.uint8), np.zeros(10, np.uint8))
    after = [[x.clone() if x is not None else None for x in before[0]]]
    hyper = dict(HYPER, eps=0.0)
    ms, vs, firsts = run(A, after, [(zeros, zeros)], [0.0], step=1, **hyper)
    zero = (grad == 0)
    assert bool(torch.isnan(after[0][0][zero]).all()) and int((~zero).sum()) > 400  # (0 / 0, as without eps it is)
    codes, nw, ew = reference(*before[0][:2], zeros, zeros, None, 0.0, 1.0, seed=7, first=0, step=1, **hyper)
    keep = ~zero.cpu().numpy()
    assert (np.abs(after[0][0].double().cpu().numpy() - nw)[keep] <= ew[keep]).all()
    for x, y in zip(ms[0] + vs[0], codes):
        assert np.array_equal(x.cpu().numpy(), y)


@pytest.mark.parametrize("bad", [math.inf, math.nan])
def test_factor_or_step_that_changes_nothing(bad):
    import paper_2503_01066_amd as A
    t = make([5000, 3], "bf16", True, 2)
    old = [[x.clone() for x in y] for y in t]
    s = [state(n, n, -7) for n in (5000, 3)]
    for kw in (dict(grad_factor=torch.full((1,), bad, device="cuda")), dict(schedule=torch.tensor([0.1, 0.0], device="cuda")),
               dict(schedule=torch.tensor([0.1, math.nan], device="cuda"))):
        ms, vs, _ = run(A, t, s, [0.1, 0.1], step=2, **kw, **HYPER)
        assert all(torch.equal(a, b) for x, y in zip(t, old) for a, b in zip(x, y))
        for i in range(2):
            assert all(np.array_equal(a.cpu().numpy().reshape(-1), b) for a, b in zip(ms[i] + vs[i], s[i][0] + s[i][1]))


def test_rounding_is_unbiased_and_second_moments_move():
    """A moment that no code holds is held on average: over n elements the mean is within 5 standard deviations of at most half a code.  v decays where
    the nearest code would hold it for ever, and none of it becomes 0."""
    import paper_2503_01066_amd as A
    n = 1 << 20
    p, z = torch.zeros(n, device="cuda"), lambda: A.adamw8_state(n)
    grad = torch.full((n,), 0.3, device="cuda")
    grad[::64] = 1.0   # (the block's largest)
    m, v = z(), z()
    A.alch_adamw8_step(A.Adamw8List([p], [grad], [m], [v]), 0.1, beta1=0.9, beta2=0.999, step=1)
    sel = np.arange(n) % 64 != 0
    f = lambda pair, which: decode(pair[0].cpu().numpy(), pair[1].cpu().numpy(), which)[sel].astype(np.float64)
    for x, true in ((f(m, "m"), 0.03), (f(v, "v"), 0.09e-3)):
        assert len(np.unique(x)) == 2 and abs(x.mean() / true - 1) <= 5 * 0.0625 / math.sqrt(len(x)), (x.mean(), true)
    before = f(v, "v")
    grad.zero_()
    for step in range(2, 202):
        A.alch_adamw8_step(A.Adamw8List([p], [grad], [m], [v]), 0.1, beta1=0.9, beta2=0.999, step=step)
    after = f(v, "v")
    # each step keeps 0.999 of the mean, with a variance of at most a quarter of a code's square an element and step
    assert abs(after.mean() / (before.mean() * 0.999 ** 200) - 1) <= 5 * 0.0625 * math.sqrt(200) / math.sqrt(len(after))
    grad[::64] = 1e4
    A.alch_adamw8_step(A.Adamw8List([p], [grad], [m], [v]), 0.1, step=300)
    assert bool((v[0] > 0).all()) and bool(torch.isfinite(p).all())


def test_schedule_captured_and_replayed():
    import paper_2503_01066_amd as A
    sizes = [3000, 9, 70000]
    start = make(sizes, "bf16", True, 4)
    copies = [[x.clone() for x in t] for t in start]
    ms, vs = [A.adamw8_state(n) for n in sizes], [A.adamw8_state(n) for n in sizes]
    l = A.Adamw8List([t[0] for t in copies], [t[1] for t in copies], ms, vs, masters=[t[2] for t in copies], weight_decay=0.01)
    schedule, factor = torch.zeros(2, device="cuda"), torch.ones(1, device="cuda")
    call = lambda: A.alch_adamw8_step(l, 0.0, seed=123, schedule=schedule, grad_factor=factor)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    def all_of():
        return [x.clone() for t in copies for x in t] + [x.clone() for s in ms + vs for x in s]
    runs = []
    for how in (call, graph.replay, graph.replay):
        for t, s in zip(copies, start):
            for x, y in zip(t, s):
                x.copy_(y)
        for s in ms + vs:
            s[0].zero_(), s[1].zero_()
        got = []
        for k in range(1, 4):
            schedule.copy_(torch.tensor([1e-2 / k, float(k)]))
            factor.fill_(1.0 / k)
            torch.cuda.synchronize()
            how()
            torch.cuda.synchronize()
            got.append(all_of())
        runs.append(got)
    for other in runs[1:]:
        assert all(torch.equal(a, b) for x, y in zip(runs[0], other) for a, b in zip(x, y))
    # and the same codes as with the step given by the call
    for t, s in zip(copies, start):
        for x, y in zip(t, s):
            x.copy_(y)
    for s in ms + vs:
        s[0].zero_(), s[1].zero_()
    A.alch_adamw8_step(l, 1e-2, seed=123, step=1, stream=torch.cuda.current_stream())
    assert all(torch.equal(a, b) for a, b in zip(all_of()[9:], runs[0][0][9:]))


def test_tensors_beyond_32_bit_offsets():
    import paper_2503_01066_amd as A
    n = (1 << 31) + 12345
    p, g = torch.zeros(n, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    m, v = A.adamw8_state(n), A.adamw8_state(n)
    g[n - 3:] = 2.0
    g[5] = 2.0
    A.alch_adamw8_step(A.Adamw8List([p], [g], [m], [v]), 0.125)
    assert p[n - 4:].tolist() == [0.0, -0.125, -0.125, -0.125] and p[5] == -0.125 and int((p != 0).sum()) == 4
    assert int((m[0] != 0).sum()) == 4 and int((v[0] != 0).sum()) == 4


@pytest.mark.parametrize("dtype,master", [("f32", False), ("bf16", False), ("bf16", True), ("f32", True)])
@pytest.mark.parametrize("base", [0, 1024, 2048, 3 * 1024, 4096, 8192])
def test_ends_in_every_wavefront_of_a_round(dtype, master, base):
    """Rounds are of 1024 or 2048 elements, a wavefront's part of 256 or 512, blocks of 64: ends beside each, whole wavefronts before them; and what lies
    behind a tensor in its memory stays."""
    import paper_2503_01066_amd as A
    sizes = sorted({max(base + k * w + e, 1) for w in (256, 512) for k in range(5) for e in (-65, -1, 0, 1, 8, 64, 100)})
    before = make(sizes, dtype, master, base)
    states = [state(n, i, -7) for i, n in enumerate(sizes)]
    roomy = lambda x, fill: torch.cat([x, torch.full((64,), fill, dtype=x.dtype, device="cuda")])
    kept = [[None if x is None else roomy(x, 9) for x in t] for t in before]
    after = [[None if x is None else x[:n] for x in t] for n, t in zip(sizes, kept)]
    dev = lambda a: roomy(torch.from_numpy(a).cuda(), 99)
    held = [[(dev(c), dev(s)) for c, s in st] for st in states]
    cut = lambda k: [(h[k][0][:n], h[k][1][:-(-n // 64)]) for n, h in zip(sizes, held)]
    masters = [t[2] for t in after] if master else None
    for lo in range(0, len(sizes), 40):  # (few tensors, whose table is in registers)
        part = slice(lo, lo + 40)
        l = A.Adamw8List([t[0] for t in after[part]], [t[1] for t in after[part]], cut(0)[part], cut(1)[part], masters=masters and masters[part], weight_decay=0.1)
        A.alch_adamw8_step(l, seed=7, step=3, **HYPER)
        firsts = [r.first for r in l.host][:len(sizes[part])]
        torch.cuda.synchronize()
        check(before[part], states[part], after[part], cut(0)[part], cut(1)[part], firsts, [0.1] * 40, None, seed=7, step=3, **HYPER)
    for n, t, h in zip(sizes, kept, held):
        assert all(x is None or bool((x[n:] == 9).all()) for x in t)
        for c, s in h:
            assert bool((c[n:] == 99).all()) and bool((s[-(-n // 64):] == 99).all())
