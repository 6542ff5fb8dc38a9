"""The clipped policy loss with its KL term against its formulas in 64 bits.

Tolerances count roundings, u = 2^-24.  With R the largest distance of a logit that matters from the row's largest one (beyond 40 a term is
below 2^-57 of the sum): a term exp(x - base) has the difference's rounding and the product with log2 e's, at most 2 u R log2 e on the
exponent, and 4 u for the exponential itself; a sum of V terms by 1024 threads or more, whose partial sums are at most V / 1024 + 16 terms long and then
joined in 16 steps, (V / 1024 + 32) u: E = u (2 * 1.45 R + 4 + V / 1024 + 32).  logp has E and three roundings of numbers of its size.  A
gradient d (onehot - p) has p E for its own exponential and for the sum, d's relative error and its rounding to the storage type; d = w (...) has
the ratio's error E' = (error of logp) + 4 u, on |A| ratio, and the KL term's the same on exp(ref - logp)."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
U = 2.0 ** -24
LOW, HIGH, KL = 0.2, 0.3, 0.07


def make(n, V, dtype, seed, std=3.0, pad=0, kl=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    f = lambda *s: torch.randn(s, generator=g, device="cuda")
    wide = (f(n, V + pad) * std).to(DT[dtype])
    x = wide[:, :V]
    label = torch.randint(0, V, (n,), generator=g, device="cuda", dtype=torch.int32)
    x.scatter_(1, label.long()[:, None], (math.log(V) + std + f(n, 1)).to(DT[dtype]))
    logp = torch.log_softmax(x.double(), 1).gather(1, label.long()[:, None])[:, 0]
    step = (f(n) * 12).round() / 100  # (whole hundredths: no ratio on a bound, log 0.8 = -0.2231, log 1.3 = 0.2624)
    return dict(x=x, label=label, old=(logp - step).float(), adv=f(n), weight=f(n).abs() + 0.1, ref=(logp + 0.3 * f(n)).float() if kl else None)


def formula(x, label, old, adv, weight, ref, kl_coef=KL, low=LOW, high=HIGH):
    """(loss [4], logp, dlogits) in 64 bits, and what the tolerances are made of."""
    x, V = x.double(), x.shape[1]
    x = x - x.max(1, keepdim=True).values  # (64 bits lose the logarithm of a sum beside a logit of 1e38)
    counted = (label >= 0) & (label < V) & (weight != 0)
    safe = label.long().clamp(0, V - 1)
    logz = torch.logsumexp(x, 1)
    logp = x.gather(1, safe[:, None])[:, 0] - logz
    w, A = weight.double() * counted, adv.double()
    ratio = torch.exp(logp - old.double())
    cut = ((A > 0) & (ratio > 1 + high)) | ((A < 0) & (ratio < 1 - low))
    s = torch.where(cut, ratio.clamp(1 - low, 1 + high), ratio) * A
    kl, grown = torch.zeros_like(w), torch.zeros_like(w)
    if ref is not None:
        far = ref.double() - logp
        grown = torch.expm1(far)
        kl = grown - far
    d = w * (-torch.where(cut, torch.zeros_like(s), ratio * A) - kl_coef * grown)
    p = torch.exp(x - logz[:, None])
    dx = -d[:, None] * p
    dx.scatter_add_(1, safe[:, None], d[:, None])
    zero = lambda t: torch.where(counted, t, torch.zeros_like(t))
    loss = torch.stack([(w * zero(-s + kl_coef * kl)).sum(), (w * zero(-s)).sum(), (w * zero(kl)).sum(), (w * (cut & counted)).sum()])
    return loss, zero(logp), torch.where(counted[:, None], dx, torch.zeros_like(dx)), dict(
        p=p, d=zero(d), w=w, ratio=zero(ratio * A.abs()), kl=zero(kl_coef * (grown + 1)), logz=logz, counted=counted, s=zero(s), k=zero(kl),
        R=(x.max(1).values - x.min(1).values).clamp(max=40.0))


def check(A, c, kl_coef=KL, low=LOW, high=HIGH, grad=True, **kw):
    it = A.PolicyItems(c["label"], c["old"], c["adv"], c["weight"], ref_logp=c["ref"])
    want, wlogp, wdx, t = formula(**c, kl_coef=kl_coef, low=low, high=high)  # (before the call, which may be in place)
    loss, logp, dx = A.alch_policy_loss(c["x"], it, clip_low=low, clip_high=high, kl_coef=kl_coef, want_grad=grad, **kw)
    torch.cuda.synchronize()
    V = c["x"].shape[1]
    E = U * (2.9 * t["R"] + 36 + V / 1024)
    el = E + 3 * U * (wlogp.abs() + t["R"] + t["logz"].abs())
    assert bool(((logp.double() - wlogp).abs() <= el).all()), float(((logp.double() - wlogp).abs() / el).max())
    er = el + 4 * U
    ed = t["w"] * (t["ratio"] * er + t["kl"] * er + 4 * U * (t["ratio"] + t["kl"])) + 2 * U * t["d"].abs()
    terms = t["w"] * (t["ratio"] * er + 4 * U * t["s"].abs())
    kls = t["w"] * ((t["kl"] / kl_coef if kl_coef else 0 * t["k"]) * er + 4 * U * (t["k"] + 1))
    bounds = torch.stack([(terms + kl_coef * kls).sum(), terms.sum(), kls.sum(), 0 * terms.sum()]) + U * want.abs() * 2
    assert bool(((loss.double() - want).abs() <= bounds).all()), (loss, want, bounds)
    if grad:
        bound = (ed + t["d"].abs() * 8 * U)[:, None] * t["p"] + 2 * E[:, None] * t["d"].abs()[:, None] * t["p"]
        own = torch.zeros_like(bound).scatter_add_(1, c["label"].long().clamp(0, V - 1)[:, None], (ed + t["d"].abs() * (el + 4 * U))[:, None])
        bound = bound + own
        bound = bound + torch.finfo(dx.dtype).eps / 2 * (wdx.abs() + bound) + 1e-44
        bad = (dx.double() - wdx).abs() > bound
        assert not bool(bad.any()), (torch.nonzero(bad)[:3], dx[bad][:3], wdx[bad][:3])
        assert bool((dx[~t["counted"]] == 0).all())
    return loss, logp, dx


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,V", [(1, 1), (3, 2), (5, 7), (4, 1000), (300, 1001), (17, 8192), (2, 16384), (33, 32003), (260, 50257), (7, 65536), (5, 128256), (3, 131071),
                                 (2, 131080), (270, 131072), (5, 151936), (2, 262147)])
def test_sizes(dtype, n, V):
    import paper_2503_01066_amd as A
    if n * V > 40e6:
        n = max(int(40e6) // V, 1)
    check(A, make(n, V, dtype, n + V))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_rows_of_a_long_vocabulary(dtype):
    """More rows than compute units, so that a work-group that stays has several."""
    import paper_2503_01066_amd as A
    c = make(700, 128256 if dtype == "bf16" else 32000, dtype, 5)
    c["weight"][torch.rand(700, device="cuda") < 0.4] = 0
    a = check(A, c)
    b = check(A, c, logp=torch.empty(700, device="cuda"), dlogits=torch.full_like(c["x"], 9.0))
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    x = c["x"].clone()
    it = A.PolicyItems(c["label"], c["old"], c["adv"], c["weight"], ref_logp=c["ref"])
    loss, logp, dx = A.alch_policy_loss(x, it, clip_low=LOW, clip_high=HIGH, kl_coef=KL, dlogits=x)  # in place
    assert dx is x and torch.equal(x, a[2]) and torch.equal(loss, a[0]) and torch.equal(logp, a[1])
    f = check(A, c, grad=False)  # (its sums are taken in another order: within the same bounds, not to the bit)
    assert f[2] is None


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,pad", [(1000, 24), (1001, 3), (32000, 1), (128250, 6), (9, 0)])
def test_rows_further_apart_than_the_vocabulary(dtype, V, pad):
    import paper_2503_01066_amd as A
    c = make(9, V, dtype, 3, pad=pad)
    wide = torch.full((9, V + 5), 9.0, dtype=DT[dtype], device="cuda")
    check(A, c, dlogits=wide[:, :V])
    assert bool((wide[:, V:] == 9.0).all())
    store = torch.full((9, V + pad), 9.0, dtype=DT[dtype], device="cuda")
    store[:, :V] = c["x"]
    # in place (the order of a row's sum goes by where it begins, so that the bits of rows elsewhere may be others)
    view = store[:, :V]
    _, _, dx = check(A, dict(c, x=view), dlogits=view)
    assert dx is view and bool((store[:, V:] == 9.0).all())


@pytest.mark.parametrize("dtype,V", [("bf16", 5000), ("f32", 5000), ("bf16", 128256), ("f32", 70001)])
def test_items_that_score_nothing_and_forbidden_tokens(dtype, V):
    import paper_2503_01066_amd as A
    c = make(40, V, dtype, 8)
    c["label"][:6] = torch.tensor([-1, V, V + 5, -2 ** 31, 2 ** 31 - 1, 0], dtype=torch.int32, device="cuda")
    c["weight"][7:9] = 0
    c["x"][0] = math.nan     # (of an item that does not score: not looked at)
    c["x"][7] = math.inf
    clean = dict(c, x=c["x"].clone())
    clean["x"][0] = clean["x"][7] = 0
    got = A.alch_policy_loss(c["x"], A.PolicyItems(c["label"], c["old"], c["adv"], c["weight"], ref_logp=c["ref"]), clip_low=LOW, clip_high=HIGH, kl_coef=KL)
    want = check(A, clean)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    # half of the vocabulary is forbidden, the label among the other half
    d = make(40, V, dtype, 9)
    keep = d["x"].gather(1, d["label"].long()[:, None])
    d["x"][:, ::2] = -math.inf
    d["x"].scatter_(1, d["label"].long()[:, None], keep)
    _, _, dx = check(A, dict(d, x=d["x"].clamp(min=torch.finfo(DT[dtype]).min)))
    got = A.alch_policy_loss(d["x"], A.PolicyItems(d["label"], d["old"], d["adv"], d["weight"], ref_logp=d["ref"]), clip_low=LOW, clip_high=HIGH, kl_coef=KL)
    assert torch.equal(got[2], dx)
    # rows without any token, with a NaN, with +inf, and a label that is forbidden itself
    e = make(8, V, dtype, 10, kl=False)
    e["x"][0] = -math.inf
    e["x"][1, V // 2] = math.nan
    e["x"][2, 3] = math.inf
    e["x"][3, e["label"][3].item()] = -math.inf
    e["x"][4] = math.nan
    run = lambda c_: A.alch_policy_loss(c_["x"], A.PolicyItems(c_["label"], c_["old"], c_["adv"], c_["weight"]), clip_low=LOW, clip_high=HIGH)
    loss, logp, dx = run(e)
    assert logp[0] == -math.inf and bool((dx[0] == 0).all()) and logp[3] == -math.inf and bool((dx[3] == 0).all())
    for r in (1, 2, 4):
        assert math.isnan(logp[r]) and bool(torch.isnan(dx[r]).all()), r
    assert math.isnan(loss[0]) and bool(torch.isfinite(dx[5:]).all())
    fine = [0, 3, 5, 6, 7]
    loss, logp, _ = run({k: v[fine].contiguous() if v is not None else None for k, v in e.items()})
    assert bool(torch.isfinite(loss).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,V", [(3, 5000), (3, 128256), (300, 2000), (600, 40000), (300, 100000)])
def test_rows_of_the_lowest_value_and_of_huge_ones(dtype, n, V):
    """Finite logits of any size have a distribution: a row all of whose tokens were masked with the type's lowest value is uniform, one among
    masked ones has all of it, and the difference of large logits counts, not their size."""
    import paper_2503_01066_amd as A
    c = make(n, V, dtype, 2)
    low, at = torch.finfo(DT[dtype]).min, c["label"].long()[:, None]
    c["x"][0] = low
    c["x"][1] = low
    c["x"][1].scatter_(0, at[1], 3.0)
    c["x"][2, : V // 2] = low
    for r, by in ((n // 2, 3e5), (n // 2 + 1, -3e5), (n - 2, 1e30), (n - 1, -1e30)):
        if r > 2:
            c["x"][r] = by
    logp = torch.log_softmax(c["x"].double(), 1).gather(1, at)[:, 0]
    c["old"], c["ref"] = (logp + 0.05).float(), (logp - 0.1).float()
    _, got, dx = check(A, c)
    assert abs(got[0].item() + math.log(V)) <= 1e-5 and got[1].item() == 0.0 and bool((dx[1] == 0).all())
    f = A.alch_policy_loss(c["x"], A.PolicyItems(c["label"], c["old"], c["adv"], c["weight"], ref_logp=c["ref"]), clip_low=LOW, clip_high=HIGH, kl_coef=KL, want_grad=False)
    assert bool(((f[1].double() - logp).abs() <= 1e-5 * (1 + logp.abs())).all())


def test_clipping_and_its_bounds():
    """Either sign of the advantage, on either side of the bounds; none; and the advantage 0 whatever the ratio."""
    import paper_2503_01066_amd as A
    c = make(12, 500, "f32", 4)
    logp = torch.log_softmax(c["x"].double(), 1).gather(1, c["label"].long()[:, None])[:, 0]
    ratio = torch.tensor([0.5, 0.9, 1.1, 2.0] * 3, device="cuda", dtype=torch.float64)
    c["old"] = (logp - ratio.log()).float()
    c["adv"] = torch.tensor([1.0] * 4 + [-1.0] * 4 + [0.0] * 4, device="cuda")
    c["weight"] = torch.full((12,), 0.25, device="cuda")
    c["ref"] = None
    loss, _, dx = check(A, c, kl_coef=0.0)
    zero = [bool((dx[i] == 0).all()) for i in range(12)]
    assert zero == [False, False, False, True, True, False, False, False] + [True] * 4 and loss[3].item() == 0.5
    want = -0.25 * (0.5 + 0.9 + 1.1 + 1.3 - 0.8 - 0.9 - 1.1 - 2.0)
    assert abs(loss[0].item() - want) <= 1e-5 and loss[0] == loss[1] and loss[2] == 0
    free = check(A, c, kl_coef=0.0, low=math.inf, high=math.inf)
    assert free[0][3] == 0 and not any(bool((free[2][i] == 0).all()) for i in range(8))
    tight = check(A, c, kl_coef=0.0, low=0.0, high=0.0)
    assert tight[0][3].item() == 1.0
    c["old"][8:] = -200.0  # (a ratio of e^190: infinite in fp32)
    loss, _, dx = A.alch_policy_loss(c["x"], A.PolicyItems(c["label"], c["old"], c["adv"], c["weight"]))
    assert bool(torch.isfinite(loss).all()) and bool((dx[8:] == 0).all())


def test_kl_alone_and_measured_only():
    import paper_2503_01066_amd as A
    c = make(50, 777, "f32", 6)
    zero = check(A, c, kl_coef=0.0)
    with_kl = check(A, c)
    assert torch.equal(zero[0][1:], with_kl[0][1:]) and zero[0][0] == zero[0][1] and with_kl[0][2] > 0
    c["adv"] = torch.zeros(50, device="cuda")
    loss, _, dx = check(A, c, kl_coef=2.0)
    assert loss[1] == 0 and not bool((dx == 0).all())
    c["ref"] = torch.log_softmax(c["x"].double(), 1).gather(1, c["label"].long()[:, None])[:, 0].float()
    loss, _, _ = check(A, c)
    assert abs(loss[2].item()) <= 1e-9  # (the reference model itself: kl is of second order in a rounding)


def test_gradient_against_differences():
    import paper_2503_01066_amd as A
    c = make(6, 90, "f32", 2)
    _, _, dx = A.alch_policy_loss(c["x"], A.PolicyItems(c["label"], c["old"], c["adv"], c["weight"], ref_logp=c["ref"]), clip_low=LOW, clip_high=HIGH, kl_coef=KL)
    way = torch.randn(6, 90, device="cuda", dtype=torch.float64)
    h = 1e-6
    loss = lambda s: formula(**dict(c, x=c["x"].double() + s * h * way))[0][0].item()
    measured = (loss(1) - loss(-1)) / (2 * h)
    # (64-bit losses of size 10 over 2e-6 leave 1e-9; the fp32 gradient's 540 elements their relative 1e-5 at most)
    assert abs(measured - float((dx.double() * way).sum())) <= 1e-8 + 1e-5 * float((dx.double() * way).abs().sum())


def test_no_items():
    import paper_2503_01066_amd as A
    e, z = torch.empty(0, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda")
    loss, logp, dx = A.alch_policy_loss(torch.empty((0, 50), device="cuda"), A.PolicyItems(z, e, e, e))
    assert loss.tolist() == [0, 0, 0, 0] and dx.shape == (0, 50)


def test_another_stream_and_captured():
    import paper_2503_01066_amd as A
    cases = {(n, V): [make(n, V, "bf16", k) for k in range(3)] for n, V in ((9, 128256), (400, 5001))}
    for (n, V), inputs in cases.items():
        c = {k: v.clone() for k, v in inputs[0].items()}
        it = A.PolicyItems(c["label"], c["old"], c["adv"], c["weight"], ref_logp=c["ref"])
        ws, s = torch.empty(A.policy_loss_workspace_bytes(n, V), dtype=torch.uint8, device="cuda"), torch.cuda.Stream()
        dx = torch.empty_like(c["x"])
        call = lambda **kw: A.alch_policy_loss(c["x"], it, kl_coef=KL, **kw)
        s.wait_stream(torch.cuda.current_stream())
        call(stream=s)
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = call(workspace=ws, dlogits=dx)
        for k in (0, 1, 2, 1):
            for key, v in inputs[k].items():
                c[key].copy_(v)
            ws.fill_(0xff)
            torch.cuda.synchronize()
            want, other = call(), call(stream=s)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) and torch.equal(a, o) for a, b, o in zip(want, got, other)), (n, V, k)


def test_refusals():
    import paper_2503_01066_amd as A
    c = make(5, 64, "bf16", 1)
    it = A.PolicyItems(c["label"], c["old"], c["adv"], c["weight"])
    for call in (lambda: A.alch_policy_loss(c["x"][:4], it), lambda: A.alch_policy_loss(c["x"].t().contiguous().t(), it),
                 lambda: A.alch_policy_loss(c["x"], it, dlogits=torch.empty(5, 64, device="cuda")), lambda: A.alch_policy_loss(c["x"], it, logp=torch.empty(4, device="cuda")),
                 lambda: A.alch_policy_loss(c["x"], it, loss=torch.empty(1, device="cuda")), lambda: A.alch_policy_loss(c["x"].cpu(), it)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(A.AlchError, match="ref_logp"):
        A.alch_policy_loss(c["x"], it, kl_coef=0.1)
    with pytest.raises(A.AlchError, match="workspace"):
        A.alch_policy_loss(c["x"], it, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))


def test_offsets_beyond_32_bits():
    import paper_2503_01066_amd as A
    n, V = 17000, 128256  # 2.18e9 logits
    x = torch.zeros((n, V), dtype=torch.bfloat16, device="cuda")
    f = lambda v: torch.full((n,), v, device="cuda")
    label = torch.full((n,), V - 1, dtype=torch.int32, device="cuda")
    weight = f(0.0)
    weight[-1] = weight[3] = 1.0
    x[-1, V - 1] = 5.0
    dx = torch.full_like(x, 9.0)
    loss, logp, _ = A.alch_policy_loss(x, A.PolicyItems(label, f(-math.log(V)), f(1.0), weight), dlogits=dx)
    p = math.exp(5) / (V - 1 + math.exp(5))
    assert abs(logp[-1].item() - math.log(p)) <= 1e-5 and abs(logp[3].item() + math.log(V)) <= 1e-5
    assert bool((dx[4:-1] == 0).all()) and bool((dx[:3] == 0).all()) and bool((dx[-1] == 0).all())  # (the last item's ratio is clipped)
    assert abs(dx[3, 0].item() * V - 1) <= 2 ** -8 and abs(dx[3, V - 1].item() + 1) <= 2 ** -8


@pytest.mark.parametrize("dtype,V", [("bf16", 65600), ("bf16", 131001), ("f32", 32808)])
@pytest.mark.parametrize("n", [257, 700, 4500])
@pytest.mark.parametrize("pattern", ["none", "all", "last", "first half", "every other", "a tenth not"])
def test_which_rows_of_a_long_vocabulary_score(dtype, V, n, pattern):
    """Rows are dealt to the work-groups by whether they score, 4096 of them at a time."""
    import paper_2503_01066_amd as A
    c = make(n, V, dtype, n)
    at = torch.arange(n, device="cuda")
    scores = {"none": at < 0, "all": at >= 0, "last": at == n - 1, "first half": at < n // 2, "every other": at % 2 == 1,
              "a tenth not": torch.rand(n, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3)) > 0.1}[pattern]
    c["weight"][~scores & (at % 3 != 0)] = 0
    c["label"][~scores & (at % 3 == 0)] = -1
    check(A, c)


def test_more_rows_than_the_work_groups_of_a_launch_have_lists_for():
    """34 GB of logits, in place: 1023 rows a compute unit are a launch.  All logits are 0, so that p = 1 / V, a power of two's neighbour: -d / V."""
    import paper_2503_01066_amd as A
    V, n = 65544, 1023 * torch.cuda.get_device_properties(0).multi_processor_count + 300
    if torch.cuda.mem_get_info()[0] < n * V * 2 + (4 << 30):
        pytest.skip("needs %d GB of device memory" % (n * V * 2 >> 30))
    x = torch.zeros(n, V, dtype=torch.bfloat16, device="cuda")
    at = torch.arange(n, device="cuda")
    label, weight = (at * 7919 % V).int(), torch.ones(n, device="cuda")
    weight[at % 5 == 2] = 0
    old, adv = torch.full((n,), -math.log(V), device="cuda"), 1.0 + at.float() / n
    loss, logp, dx = A.alch_policy_loss(x, A.PolicyItems(label, old, adv, weight), dlogits=x)
    counted = weight != 0
    # ln V = 11.1: its rounding, that of the sum (V / 1024 + 32 additions) and of the logarithm; old's own
    e = U * (V / 1024 + 36 + 6 * 11.1)
    assert bool((logp[counted].double() + math.log(V)).abs().max() <= e) and bool((logp[~counted] == 0).all())
    for b in range(0, n, 8192):
        got, lab, c = dx[b:b + 8192], label[b:b + 8192].long(), counted[b:b + 8192]
        d = torch.where(c, -adv[b:b + 8192], torch.zeros(1, device="cuda")).double()
        assert bool(((got.gather(1, lab[:, None])[:, 0].double() - d * (1 - 1 / V)).abs() <= (2.0 ** -8 + 2 * e) * d.abs()).all())
        got.scatter_(1, lab[:, None], 0)
        most, least = got.amax(1).double(), got.masked_fill(torch.zeros_like(got, dtype=torch.bool).scatter_(1, lab[:, None], True), 1.0).amin(1).double()
        for side in (most, least):
            assert bool(((side[c] + d[c] / V).abs() <= (2.0 ** -8 + 3 * e) * d[c].abs() / V).all())
        assert bool((most[~c] == 0).all()) and bool((got[~c].amin(1) == 0).all())


@pytest.mark.parametrize("dtype,V", [("bf16", 131080), ("bf16", 204800), ("bf16", 204808), ("bf16", 230001), ("f32", 65540), ("f32", 102400), ("f32", 102404),
                                     ("f32", 128256), ("f32", 150003)])
def test_rows_that_registers_do_not_hold(dtype, V):
    """Registers hold 16 pieces of 16 bytes a thread of 1024, LDS 9 more, the rest is read again: the label, the largest logit, forbidden
    tokens, the type's lowest value and NaN on every side of the borders."""
    import paper_2503_01066_amd as A
    c = make(336, V, dtype, V)
    per = 1024 * (8 if dtype == "bf16" else 4)
    at = sorted({min(max(e, 0), V - 1) for b in (0, 16 * per, 25 * per, V) for e in (b - 1, b, b + 9)})
    c["label"][:len(at)] = torch.tensor(at, dtype=torch.int32, device="cuda")
    for i, e in enumerate(at):
        c["x"][20 + i, e] = 60.0                   # the largest one
        c["x"][40 + i, :e] = -math.inf             # nothing before,
        c["x"][40 + i, e] = 1.0
        c["x"][60 + i, e + 1:] = -math.inf         # nothing behind
        c["x"][60 + i, e] = 1.0
        c["x"][80 + i] = torch.finfo(DT[dtype]).min
        c["x"][80 + i, e] = 3.0
        c["x"][100 + i, e:] = 3e38                 # (so large that no power of two scales them)
        c["label"][100 + i] = c["label"][40 + i] = V - 1
        c["label"][60 + i], c["label"][80 + i] = 0, e
        if e > 0:
            c["x"][60 + i, 0] = 2.0
    safe = torch.where(torch.isfinite(c["x"][:120]), c["x"][:120].double(), torch.full((), -1e300, dtype=torch.float64, device="cuda"))
    logp = torch.log_softmax(safe - safe.amax(1, keepdim=True), 1).gather(1, c["label"][:120].long()[:, None])[:, 0]
    c["old"][:120], c["ref"][:120] = (logp + 0.03).float(), (logp - 0.1).float()  # (ratios near 1 whatever was planted)
    c["weight"][200:220] = 0
    check(A, c)
    c["x"][120] = -math.inf
    for i, e in enumerate(at):
        c["x"][130 + i, e] = math.nan
    items = A.PolicyItems(c["label"], c["old"], c["adv"], c["weight"], ref_logp=c["ref"])
    loss, logp, dx = A.alch_policy_loss(c["x"], items, clip_low=LOW, clip_high=HIGH, kl_coef=KL)
    assert logp[120].item() == -math.inf and bool((dx[120] == 0).all()) and math.isnan(loss[0].item())
    nan = torch.isnan(dx)
    assert bool(nan[130:130 + len(at)].all()) and not bool(nan[:130].any()) and not bool(nan[130 + len(at):].any())
