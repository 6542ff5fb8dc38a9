"""The two ends of a training step, as cases that can be made, run and compared: the embedding rows in front of the first
layer and their gradient behind it, the norm of all gradients with their clipping, and the update of the weights.

A case is a dict of plain values.  `listed()` gives the fixed ones, `draw()` more of the same ranges, `prepare()` makes what
a user's program holds before the call, `run()` is one pass (with `own` through the package's entry points, without it in
plain torch operations), `work()` the bytes and operations no implementation can do without, `exact()` the outputs in 64 bits.

Four kinds of pass ("op"):
  embed   X[t] = scale * W[id_t], a zero row where id_t is no row of W (padding)
  scatter dW[v] (+)= scale * sum of dX[t] over the tokens with id_t = v
  clip    the 2-norm over all gradients, and every gradient times min(1, max_norm / norm)
  adamw   one AdamW update of all parameters from gradients times a factor held on the device
The tensors of the last two are views of one flat buffer each, as a program with many of them keeps them; those with weight
decay come first.
"""
import math

import numpy as np
import torch

own = False

BETA1, BETA2, EPS, LR, DECAY, STEP = 0.9, 0.95, 1e-8, 3e-4, 0.1, 1000
PAD = 8  # elements: every tensor in a flat buffer starts at a multiple of 16 bytes


def listed():
    return [
        # the newest token of one sequence while it is served: latency alone
        dict(name="embed one token", op="embed", tokens=1, hidden=4096, vocab=128256, dtype="bf16", scale=1.0, padding=0.0),
        # long fp32 prompts, rows of 1948 bytes: not made of 16-byte pieces; the last tokens are padding
        dict(name="embed odd fp32", op="embed", tokens=5003, hidden=487, vocab=1000, dtype="f32", scale=22.0, padding=0.1),
        # the serving batch in front of the first layer: 32 prompts, the last of them padded
        dict(name="embed batch", op="embed", tokens=70001, hidden=4096, vocab=128256, dtype="bf16", scale=64.0, padding=0.02),
        # one short prompt into the gradient of a table shared with the head: only the rows that occur are touched
        dict(name="scatter one prompt", op="scatter", tokens=487, hidden=4096, vocab=128256, dtype="bf16", scale=1.0, padding=0.0, accumulate=True),
        # the fp32 test model: few rows, each met often
        dict(name="scatter fp32 small table", op="scatter", tokens=5003, hidden=256, vocab=1000, dtype="f32", scale=16.0, padding=0.1, accumulate=False),
        # eight prompts of 2048 tokens, the whole gradient written
        dict(name="scatter batch", op="scatter", tokens=16384, hidden=4096, vocab=128256, dtype="bf16", scale=1.0, padding=0.0, accumulate=False),
        # gradients of one fp32 layer of the test model: latency
        dict(name="clip fp32 layer", op="clip", set="layer", hidden=256, kv=256, ffn=1024, layers=1, rank=0, dtype="f32", max_norm=0.5),
        # rank-8 adapters on all projections of 32 layers: 448 small tensors
        dict(name="clip adapters", op="clip", set="adapters", hidden=4096, kv=1024, ffn=14336, layers=32, rank=8, dtype="bf16", max_norm=1.0),
        # all nine gradients of one layer of the 8B shape
        dict(name="clip 8b layer", op="clip", set="layer", hidden=4096, kv=1024, ffn=14336, layers=1, rank=0, dtype="bf16", max_norm=1.0),
        dict(name="adamw fp32 layer", op="adamw", set="layer", hidden=256, kv=256, ffn=1024, layers=1, rank=0, dtype="f32", master=False),
        dict(name="adamw adapters", op="adamw", set="adapters", hidden=4096, kv=1024, ffn=14336, layers=32, rank=8, dtype="bf16", master=True),
        dict(name="adamw 8b layer", op="adamw", set="layer", hidden=4096, kv=1024, ffn=14336, layers=1, rank=0, dtype="bf16", master=True),
    ]


def _spread(rng, low, high):
    """A whole number, spread over the logarithm of its range."""
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op, dtype = rng.choice(["embed", "scatter", "clip", "adamw"]), rng.choice(["bf16", "bf16", "f32"])
    if op in ("embed", "scatter"):
        hidden = rng.choice([256, 2048, 4096, 5120, 8192, _spread(rng, 65, 5000)])
        vocab = _spread(rng, 1000, 128256)
        c = dict(op=op, tokens=_spread(rng, 1, 70001 if op == "embed" else 16384), hidden=hidden, vocab=min(vocab, 525336576 // hidden),
                 dtype=dtype, scale=rng.choice([1.0, 16.0, 0.37]), padding=rng.choice([0.0, 0.05, 0.5]))
        return c if op == "embed" else dict(c, accumulate=rng.random() < 0.5)
    kind = rng.choice(["layer", "adapters", "mixed"])
    hidden = 8 * _spread(rng, 32, 512)
    c = dict(op=op, set=kind, hidden=hidden, kv=hidden // 4, ffn=8 * (hidden * 7 // 16), layers=1, rank=0, dtype=dtype)
    if kind == "adapters":
        c.update(layers=rng.randint(1, 32), rank=rng.choice([8, 16, 64]))
        c["layers"] = min(c["layers"], 4 + 28 * 8 // c["rank"])
    if kind == "mixed":  # tensors of any length, most of them short
        c.update(tensors=_spread(rng, 1, 300), lengths=rng.randint(1, 1 << 20))
    return dict(c, max_norm=rng.choice([1.0, 0.1, 1e6])) if op == "clip" else dict(c, master=dtype == "bf16" and rng.random() < 0.7)


def _lengths(case):
    """Elements of every tensor, and how many of the tensors (the first ones) have weight decay."""
    H, KD, F, L, r = case["hidden"], case["kv"], case["ffn"], case["layers"], case["rank"]
    if case["set"] == "layer":
        return [H * H, KD * H, KD * H, H * H, F * H, F * H, H * F] * L + [H, H] * L, 7 * L
    if case["set"] == "adapters":
        pairs = [(H, H), (H, KD), (H, KD), (H, H), (H, F), (H, F), (F, H)]
        return [n for _ in range(L) for i, o in pairs for n in (r * i, r * o)], 14 * L
    g = np.random.RandomState(case["lengths"])
    n = [int(round(math.exp(x))) for x in g.uniform(0.0, math.log(H * H), case["tensors"])]
    return n, (len(n) + 1) // 2


def _layout(case):
    """(offset, length) of every tensor in the flat buffer, the buffer's length, and where the part without weight decay begins."""
    lengths, decayed = _lengths(case)
    at = np.concatenate([[0], np.cumsum([-(-n // PAD) * PAD for n in lengths])])
    return [(int(a), n) for a, n in zip(at, lengths)], int(at[-1]), int(at[decayed])


def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _ids(case, seed):
    """Token ids as texts have them, the n-th most frequent one met about 1/n as often as the first; padding is -1."""
    r = np.random.RandomState(seed % (1 << 31))
    T, V = case["tokens"], case["vocab"]
    rank = np.minimum(np.floor(np.exp(r.uniform(0.0, math.log(V + 1.0), T))).astype(np.int64) - 1, V - 1)
    ids = r.permutation(V)[rank]
    ids[T - int(T * case["padding"]):] = -1
    return ids.astype(np.int32)


def _normal(g, n, std, dtype):
    return torch.empty(n, dtype=dtype, device="cuda").normal_(0.0, std, generator=g)


def _filled(layout, size, g, std, dtype, make=_normal):
    """A flat buffer with zeros between the tensors."""
    flat = make(g, size, std, dtype)
    gaps = np.concatenate([np.arange(a + n, a + -(-n // PAD) * PAD) for a, n in layout])
    flat[torch.from_numpy(gaps.astype(np.int64)).cuda()] = 0
    return flat


def _square(g, n, std, dtype):
    return _normal(g, n, std, dtype).square_()


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt, s = _type(case), dict(case=case)
    if case["op"] in ("embed", "scatter"):
        T, H, V = case["tokens"], case["hidden"], case["vocab"]
        s["ids"] = torch.from_numpy(_ids(case, seed)).cuda()
        if case["op"] == "embed":
            s["W"] = _normal(g, (V, H), 0.02, dt)
            s["X"] = torch.empty((T, H), dtype=dt, device="cuda")
        else:
            s["dX"] = _normal(g, (T, H), 0.01, dt)
            s["dW"] = _normal(g, (V, H), 0.01, dt)
            if own:
                import paper_2503_01066_amd as A
                s["ws"] = torch.empty(A.embed_backward_workspace_bytes(dt, V, H, T), dtype=torch.uint8, device="cuda")
        return s
    layout, size, plain = _layout(case)
    s.update(plain=plain, grad=_filled(layout, size, g, 0.01, dt))
    parts = lambda flat: [flat[a:a + n] for a, n in layout]
    if case["op"] == "clip":
        s["out"] = torch.zeros_like(s["grad"])
        if own:
            import paper_2503_01066_amd as A
            s["list"] = A.GradList(parts(s["grad"]), parts(s["out"]))
            s["ws"] = torch.empty(A.grad_clip_workspace_bytes(), dtype=torch.uint8, device="cuda")
            s["norm"] = torch.empty(2, dtype=torch.float32, device="cuda")
        return s
    master = _filled(layout, size, g, 0.02, torch.float32)
    s.update(param=master.to(dt), m=_filled(layout, size, g, 3e-3, torch.float32), v=_filled(layout, size, g, 8e-3, torch.float32, _square),
             factor=torch.full((1,), 0.5 + 0.001 * (seed % 400), dtype=torch.float32, device="cuda"))
    if case["master"]:
        s["master"] = master
    if own:
        import paper_2503_01066_amd as A
        s["list"] = A.AdamwList(parts(s["param"]), parts(s["grad"]), parts(s["m"]), parts(s["v"]),
                                masters=parts(master) if case["master"] else None,
                                weight_decay=[DECAY if a < plain else 0.0 for a, n in layout])
    return s


def run(s):
    return {"embed": _embed, "scatter": _scatter, "clip": _clip, "adamw": _adamw}[s["case"]["op"]](s)


def _embed(s):
    c = s["case"]
    if own:
        import paper_2503_01066_amd as A
        return A.alch_embed_forward(s["ids"], s["W"], scale=c["scale"], X=s["X"])
    ids = s["ids"].long()
    rows = s["W"][ids.clamp(0, c["vocab"] - 1)].float() * c["scale"]
    s["X"].copy_(torch.where(((ids >= 0) & (ids < c["vocab"]))[:, None], rows, torch.zeros_like(rows)))
    return s["X"]


def _scatter(s):
    c = s["case"]
    if own:
        import paper_2503_01066_amd as A
        return A.alch_embed_backward(s["ids"], s["dX"], c["vocab"], scale=c["scale"], dW_embed=s["dW"], accumulate=c["accumulate"], workspace=s["ws"])
    valid = (s["ids"] >= 0) & (s["ids"] < c["vocab"])
    ids, rows = s["ids"].long()[valid], s["dX"][valid].float()
    if c["accumulate"]:  # of the rows that occur alone
        met, place = torch.unique(ids, return_inverse=True)
        sums = torch.zeros((met.numel(), c["hidden"]), dtype=torch.float32, device="cuda").index_add_(0, place, rows)
        s["dW"][met] = (s["dW"][met].float() + sums * c["scale"]).to(s["dW"].dtype)
    else:
        s["dW"].copy_(torch.zeros((c["vocab"], c["hidden"]), dtype=torch.float32, device="cuda").index_add_(0, ids, rows).mul_(c["scale"]))
    return s["dW"]


def _clip(s):
    c = s["case"]
    if own:
        import paper_2503_01066_amd as A
        return A.alch_grad_clip(s["list"], c["max_norm"], norm_out=s["norm"], workspace=s["ws"]), s["out"]
    g = s["grad"].float()
    norm = (g * g).sum(dtype=torch.float64).sqrt()  # (a long sum)
    factor = (c["max_norm"] / norm).clamp(max=1.0).float()
    s["out"].copy_(g * factor)
    return torch.stack([norm.float(), factor]), s["out"]


def _adamw(s):
    if own:
        import paper_2503_01066_amd as A
        A.alch_adamw_step(s["list"], LR, BETA1, BETA2, EPS, STEP, grad_factor=s["factor"])
    else:
        g, m, v = s["grad"].float() * s["factor"], s["m"], s["v"]
        w = s.get("master", s["param"].float())
        m.mul_(BETA1).add_(g * (1 - BETA1))
        v.mul_(BETA2).add_(g * g * (1 - BETA2))
        change = m / (1 - BETA1 ** STEP) / ((v / (1 - BETA2 ** STEP)).sqrt() + EPS)
        change[:s["plain"]] += DECAY * w[:s["plain"]]
        w -= LR * change
        s["param"].copy_(w)
    return [s["param"], s["m"], s["v"]] + ([s["master"]] if "master" in s else [])


def work(case):
    E = 2 if case["dtype"] == "bf16" else 4
    if case["op"] in ("embed", "scatter"):
        T, H, V = case["tokens"], case["hidden"], case["vocab"]
        ids = _ids(case, 1)
        ids = ids[ids >= 0]
        met = np.unique(ids).size
        if case["op"] == "embed":
            return dict(bytes=4 * T + (met + T) * H * E, flops=T * H)
        rows = 2 * met if case["accumulate"] else V
        return dict(bytes=4 * T + (ids.size + rows) * H * E, flops=(ids.size + met) * H)
    n = sum(_lengths(case)[0])
    if case["op"] == "clip":
        return dict(bytes=2 * n * E, flops=3 * n)
    return dict(bytes=n * (2 * E + 16 + (8 if case["master"] else E)), flops=15 * n)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "embed":
        out = torch.zeros((case["tokens"], case["hidden"]), dtype=torch.float64, device="cuda")
        at = torch.nonzero(s["ids"] >= 0)[:, 0]
        out[at] = s["W"].index_select(0, s["ids"][at]).double() * case["scale"]
        return out
    if case["op"] == "scatter":
        # sums of the sorted tokens as differences of a running sum
        ids, order = torch.sort(s["ids"].long(), stable=True)
        ids, order = ids[ids >= 0], order[ids >= 0]
        out = s["dW"].double() if case["accumulate"] else torch.zeros((case["vocab"], case["hidden"]), dtype=torch.float64, device="cuda")
        if ids.numel():
            total = torch.cumsum(s["dX"][order].double(), 0)
            last = torch.nonzero(torch.cat([ids[1:] != ids[:-1], torch.ones(1, dtype=torch.bool, device="cuda")]))[:, 0]
            sums = total[last]
            sums[1:] -= total[last[:-1]]
            out[ids[last]] += case["scale"] * sums
        return out
    g = s["grad"].double()
    if case["op"] == "clip":
        norm = math.sqrt(float(torch.dot(g, g)))
        factor = case["max_norm"] / norm if norm > case["max_norm"] else 1.0
        return torch.tensor([norm, factor], dtype=torch.float64, device="cuda"), g * factor
    layout, size, plain = _layout(case)
    decay = torch.zeros(size, dtype=torch.float64, device="cuda")
    decay[:plain] = DECAY
    g *= float(s["factor"])
    m = BETA1 * s["m"].double() + (1 - BETA1) * g
    v = BETA2 * s["v"].double() + (1 - BETA2) * g.square()
    w = s.get("master", s["param"]).double()
    w = w - LR * (m / (1 - BETA1 ** STEP) / (torch.sqrt(v / (1 - BETA2 ** STEP)) + EPS) + decay * w)
    return [w, m, v] + ([w] if "master" in s else [])
