"""What a program that trains beside serving keeps and learns from in fewer bits: records captured in 8 bits and read back, the
clipped policy loss on logits of served responses, and the AdamW update with moments in 8 bits.

A case is a dict of plain values.  `listed()` gives the fixed ones, `draw()` more of the same ranges, `prepare()` makes what
a user's program holds before the call, `run()` is one pass (with `own` through the package's entry points, without it in
plain torch operations), `work()` the bytes and operations no implementation can do without, `exact()` the outputs in 64 bits.

Four kinds of pass ("op"):
  pack8   the kept tokens' rows of several activations as int8 codes with a scale for every 64 elements of a row
  expand  such rows (all, or listed ones) as bf16 or fp32 tensors
  policy  log-probabilities of sampled tokens from their logits, the clipped policy loss with its KL term, the logits' gradient
  adamw8  one AdamW update of all parameters, both moments held in 8 bits with a scale for every 64 elements
Codes and the scales that are powers of two are whole numbers here: all of them are defined bit for bit, so that equal codes and equal
scales are equal values.  The plain forms therefore make each of their roundings where the definition has it.
"""
import math

import numpy as np
import torch

own = False

GROUP = 64  # elements that share a scale
BETA1, BETA2, EPS, LR, DECAY, STEP = 0.9, 0.95, 1e-8, 3e-4, 0.1, 1000
CLIP_LOW, CLIP_HIGH, KL = 0.2, 0.28, 0.05
# name -> the widths of X, Q, K, V, G and U
WIDTHS = {"8b": (4096, 4096, 1024, 1024, 14336, 14336), "phi4": (5120, 5120, 1280, 1280, 17920, 17920),
          "h2048": (2048, 2048, 512, 512, 8192, 8192), "h256": (256, 256, 256, 256, 1024, 1024)}


def listed():
    return [
        # one short query was served and a quarter of its tokens is recorded: latency
        dict(name="pack8 one prompt", op="pack8", shape="8b", seqs=1, tokens=317, keep=0.25, dtype="bf16"),
        # fp32 records of rows that are made neither of whole groups nor of 16-byte pieces
        dict(name="pack8 odd fp32", op="pack8", shape="odd", width=487, seqs=7, tokens=5003, keep=0.5, dtype="f32"),
        # one layer of a full prefill batch, six streams of 32 prompts
        dict(name="pack8 batch", op="pack8", shape="8b", seqs=32, tokens=70001, keep=0.25, dtype="bf16"),
        # the record of that short query back in bf16, in front of a layer's backward
        dict(name="expand one prompt", op="expand", shape="8b", rows=79, listed=False, dtype="bf16"),
        # four prompts of 2048 tokens out of a larger record
        dict(name="expand layer", op="expand", shape="8b", rows=8192, listed=True, dtype="bf16"),
        # a single short response: the row of each of its tokens is one long softmax
        dict(name="policy short response", op="policy", items=17, vocab=128256, dtype="bf16", masked=0.0, kl=True, grad=True),
        # fp32 logits whose rows begin at no multiple of 16 bytes, some tokens outside of the loss
        dict(name="policy odd fp32", op="policy", items=1501, vocab=32003, dtype="f32", masked=0.1, kl=True, grad=True),
        # log-probabilities and loss alone: what the sampling and the reference model need
        dict(name="policy forward", op="policy", items=6001, vocab=128256, dtype="bf16", masked=0.0, kl=False, grad=False),
        # a batch of responses with the gradient
        dict(name="policy batch", op="policy", items=6001, vocab=128256, dtype="bf16", masked=0.1, kl=True, grad=True),
        # one fp32 layer of the test model: latency
        dict(name="adamw8 fp32 layer", op="adamw8", set="layer", hidden=256, kv=256, ffn=1024, layers=1, rank=0, dtype="f32", master=False),
        # rank-8 adapters on all projections of 32 layers: 448 small tensors
        dict(name="adamw8 adapters", op="adamw8", set="adapters", hidden=4096, kv=1024, ffn=14336, layers=32, rank=8, dtype="bf16", master=True),
        # all nine tensors of one layer of the 8B shape
        dict(name="adamw8 8b layer", op="adamw8", set="layer", hidden=4096, kv=1024, ffn=14336, layers=1, rank=0, dtype="bf16", master=True),
    ]


def _spread(rng, low, high):
    """A whole number, spread over the logarithm of its range."""
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op, dtype = rng.choice(["pack8", "expand", "policy", "policy", "adamw8", "adamw8"]), rng.choice(["bf16", "bf16", "f32"])
    if op in ("pack8", "expand"):
        c = dict(op=op, shape=rng.choice(["8b", "phi4", "h2048", "h256", "odd"]), dtype=dtype)
        if c["shape"] == "odd":
            c["width"] = _spread(rng, 1, 20000)
        per_token = sum(_widths(c)) * (2 if dtype == "bf16" else 4)
        most = 70001 * 77824 // per_token
        if op == "expand":
            return dict(c, rows=_spread(rng, 1, min(20000, most // 4)), listed=rng.random() < 0.5)
        tokens = _spread(rng, 1, min(90000, most))
        c.update(tokens=tokens, seqs=min(tokens, rng.randint(1, 40)), keep=rng.choice([0.1, 0.25, 0.5, 1.0]))
        c["tokens"] = min(tokens, max(1, int(17500 * 77824 / (c["keep"] * per_token))))
        c["seqs"] = min(c["seqs"], c["tokens"])
        return c
    if op == "policy":
        vocab = rng.choice([32000, 128256, _spread(rng, 1000, 160000)])
        most = 6001 * 128256 * 2 // (vocab * (2 if dtype == "bf16" else 4))
        return dict(op=op, items=_spread(rng, 1, min(8192, most)), vocab=vocab, dtype=dtype, masked=rng.choice([0.0, 0.1, 0.6]),
                    kl=rng.random() < 0.6, grad=rng.random() < 0.8)
    kind = rng.choice(["layer", "adapters", "mixed"])
    hidden = 8 * _spread(rng, 32, 512)
    c = dict(op=op, set=kind, hidden=hidden, kv=hidden // 4, ffn=8 * (hidden * 7 // 16), layers=1, rank=0, dtype=dtype)
    if kind == "adapters":
        c.update(layers=rng.randint(1, 32), rank=rng.choice([8, 16, 64]))
        c["layers"] = min(c["layers"], 4 + 28 * 8 // c["rank"])
    if kind == "mixed":  # tensors of any length, most of them short
        c.update(tensors=_spread(rng, 1, 200), lengths=rng.randint(1, 1 << 20))
    return dict(c, master=dtype == "bf16" and rng.random() < 0.7)


# ---- sizes of a case ----------------------------------------------------------------------------------------------

def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _widths(case):
    return (case["width"], case["width"] // 3 + 1) if case["shape"] == "odd" else WIDTHS[case["shape"]]


def _groups(width):
    return -(-width // GROUP)


def _kept(case):
    return max(1, int(round(case["tokens"] * case["keep"])))


def _bounds(case):
    """Where the prompts begin and end, a function of the case alone."""
    n, total = case["seqs"], case["tokens"]
    r = np.random.RandomState(n * 100003 + total)
    inner = np.sort(r.randint(0, total + 1, n - 1))
    return np.concatenate([[0], inner, [total]]).astype(np.int32)


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
    at = np.concatenate([[0], np.cumsum([GROUP * _groups(n) for n in lengths])])
    return [(int(a), n) for a, n in zip(at, lengths)], int(at[-1]), int(at[decayed])


# ---- inputs -------------------------------------------------------------------------------------------------------

def _normal(g, size, std, dtype):
    return torch.empty(size, dtype=dtype, device="cuda").normal_(0.0, std, generator=g)


def _activations(g, rows, width, dtype):
    """Activations as layers have them: a few channels are far larger than the others."""
    x = _normal(g, (rows, width), 1.0, dtype)
    x[:, torch.randint(0, width, (1 + width // 512,), device="cuda", generator=g)] *= 20
    return x


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return {"pack8": _prepare_pack8, "expand": _prepare_expand, "policy": _prepare_policy, "adamw8": _prepare_adamw8}[case["op"]](case, seed, g)


def _prepare_pack8(case, seed, g):
    dt, T, widths, kept = _type(case), case["tokens"], _widths(case), _kept(case)
    mask = np.zeros(T, np.uint8)
    mask[np.random.RandomState(seed % (1 << 31)).permutation(T)[:kept]] = 1
    if case["shape"] == "odd":
        streams = [_activations(g, T, w, dt) for w in widths]
    else:  # query, key and value are columns of one buffer, gate and up of another
        H, QD, KD, _, F, _ = widths
        hid, qkv, gu = (_activations(g, T, w, dt) for w in (H, QD + 2 * KD, 2 * F))
        streams = [hid, qkv[:, :QD], qkv[:, QD:QD + KD], qkv[:, QD + KD:], gu[:, :F], gu[:, F:]]
    cu = _bounds(case)
    s = dict(case=case, kept=kept, streams=streams, mask=torch.from_numpy(mask).cuda(), cu=torch.from_numpy(cu).cuda(),
             dsts=[(torch.empty((kept, w), dtype=torch.int8, device="cuda"), torch.empty((kept, _groups(w)), dtype=torch.float32, device="cuda"))
                   for w in widths])
    if own:
        import paper_2503_01066_amd as A
        s["batch"] = A.Batch(cu)
        s["ws"] = torch.empty(A.lib().alch_capture_pack_workspace_bytes(T), dtype=torch.uint8, device="cuda")
    return s


def _prepare_expand(case, seed, g):
    dt, n, widths = _type(case), case["rows"], _widths(case)
    held = n + n // 2 if case["listed"] else n
    records = [(_normal(g, (held, w), 42.0, torch.float32).round_().clamp_(-127, 127).to(torch.int8), _normal(g, (held, _groups(w)), 0.3, torch.float32).exp_() * 0.02)
               for w in widths]
    rows = None
    if case["listed"]:  # the kept tokens in their order, the last of them padding
        at = np.sort(np.random.RandomState(seed % (1 << 31)).permutation(held)[:n]).astype(np.int32)
        at[n - n // 50:] = -1
        rows = torch.from_numpy(at).cuda()
    return dict(case=case, records=records, rows=rows, outs=[torch.empty((n, w), dtype=dt, device="cuda") for w in widths])


def _prepare_policy(case, seed, g):
    dt, n, V = _type(case), case["items"], case["vocab"]
    logits = _normal(g, (n, V), 2.0, dt)
    label = torch.randint(0, V, (n,), device="cuda", generator=g)
    likely = math.log(V) + 2.0 + _normal(g, (n, 1), 1.5, torch.float32)  # (a sampled token is a likely one; log V + 2 is the log-normaliser)
    logits.scatter_(1, label[:, None], likely.to(dt))
    logp = torch.cat([x.gather(1, l[:, None])[:, 0].float() - torch.logsumexp(x.float(), 1) for x, l in zip(logits.split(512), label.split(512))])
    # the steps between the two policies in whole hundredths: the gradient jumps where the ratio meets its bounds, and on either side of a
    # jump an answer is right, so that no token stands on one
    old = logp - (_normal(g, (n,), 12.0, torch.float32).round() / 100)
    counted = torch.ones(n, dtype=torch.float32, device="cuda")
    counted[torch.from_numpy(np.random.RandomState(seed % (1 << 31)).permutation(n)[:int(n * case["masked"])]).cuda()] = 0
    s = dict(case=case, logits=logits, label=label.int(), old=old, ref=logp + _normal(g, (n,), 0.2, torch.float32) if case["kl"] else None,
             advantage=_normal(g, (n,), 1.0, torch.float32), weight=counted / counted.sum().clamp(min=1.0),
             grad=torch.zeros_like(logits) if case["grad"] else None)
    if own:
        import paper_2503_01066_amd as A
        s["items"] = A.PolicyItems(s["label"], s["old"], s["advantage"], s["weight"], ref_logp=s["ref"])
        s["ws"] = torch.empty(A.policy_loss_workspace_bytes(n, V), dtype=torch.uint8, device="cuda")
        s["logp"], s["loss"] = torch.empty(n, dtype=torch.float32, device="cuda"), torch.empty(4, dtype=torch.float32, device="cuda")
    return s


def _prepare_adamw8(case, seed, g):
    dt, (layout, size, plain) = _type(case), _layout(case)
    held = torch.zeros(size, dtype=torch.bool, device="cuda")  # zeros between the tensors
    for a, n in layout:
        held[a:a + n] = True
    filled = lambda std, dtype: _normal(g, size, std, dtype).mul_(held)
    grad, master = filled(0.01, dt), filled(0.02, torch.float32)
    half = torch.full((size,), 1 << 15, dtype=torch.int32, device="cuda")
    m, v = _to_m(filled(3e-3, torch.float32), half), _to_v(filled(8e-3, torch.float32).square_(), half)
    s = dict(case=case, size=size, plain=plain, grad=grad, param=master.to(dt), m=m, v=v, seed=seed % (1 << 32),
             factor=torch.full((1,), 0.5 + 0.001 * (seed % 400), dtype=torch.float32, device="cuda"))
    if case["master"]:
        s["master"] = master
    if own:
        import paper_2503_01066_amd as A
        # codes between the tensors are nobody's, and stay; a pass over the whole buffer leaves a zero there whose sign the gradient's zero has a
        # part in
        m[0].copy_(torch.where(held, m[0], m[0] * torch.signbit(grad)))
        parts = lambda flat: [flat[a:a + n] for a, n in layout]
        states = lambda pair: [(pair[0][a:a + n], pair[1][a // GROUP:a // GROUP + _groups(n)]) for a, n in layout]
        s["list"] = A.Adamw8List(parts(s["param"]), parts(grad), states(m), states(v), masters=parts(master) if case["master"] else None,
                                 weight_decay=[DECAY if a < plain else 0.0 for a, n in layout])
    return s


# ---- one pass -----------------------------------------------------------------------------------------------------

def run(s):
    return {"pack8": _pack8, "expand": _expand, "policy": _policy, "adamw8": _adamw8}[s["case"]["op"]](s)


def _pack8(s):
    if own:
        import paper_2503_01066_amd as A
        return A.alch_capture_pack_q8(s["batch"], s["mask"], s["streams"], capacity=s["kept"], dsts=s["dsts"], workspace=s["ws"])
    keep = s["mask"] != 0
    before = torch.cumsum(torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), keep.long()]), 0)
    index = torch.nonzero(keep)[:, 0]
    for x, (codes, scales) in zip(s["streams"], s["dsts"]):
        width = x.shape[1]
        rows = torch.nn.functional.pad(x[index].float(), (0, GROUP * _groups(width) - width)).view(s["kept"], -1, GROUP)
        most = rows.abs().amax(2)
        r = torch.full_like(most, 127.0) / most
        fine, some = torch.isfinite(most), most >= 2.0 ** -100
        r = torch.where(fine & some, r, torch.zeros_like(r))
        rows = torch.where(fine[:, :, None], rows, torch.zeros_like(rows))
        codes.copy_(torch.round(rows * r[:, :, None]).view(s["kept"], -1)[:, :width])
        scale = torch.where(some, most / torch.full_like(most, 127.0), torch.zeros_like(most))
        scales.copy_(torch.where(fine, scale, torch.full_like(scale, math.nan)))
    count = before[-1:]
    return index.int(), before[s["cu"].long()].int(), torch.cat([count, (count > s["kept"]).long()]).int(), s["dsts"]


def _expand(s):
    if own:
        import paper_2503_01066_amd as A
        return A.alch_record_expand(s["records"], outs=s["outs"], rows=s["rows"])
    for (codes, scales), out in zip(s["records"], s["outs"]):
        width = codes.shape[1]
        if s["rows"] is not None:
            at = s["rows"].long().clamp(0, codes.shape[0] - 1)
            codes, scales = codes[at], scales[at]
        x = codes.float() * scales.repeat_interleave(GROUP, 1)[:, :width]
        if s["rows"] is not None:
            there = (s["rows"] >= 0) & (s["rows"] < s["records"][0][0].shape[0])
            x = torch.where(there[:, None], x, torch.zeros_like(x))
        out.copy_(x)
    return s["outs"]


def _policy(s):
    c = s["case"]
    if own:
        import paper_2503_01066_amd as A
        loss, logp, grad = A.alch_policy_loss(s["logits"], s["items"], clip_low=CLIP_LOW, clip_high=CLIP_HIGH, kl_coef=KL if c["kl"] else 0.0,
                                              want_grad=c["grad"], dlogits=s["grad"], logp=s["logp"], loss=s["loss"], workspace=s["ws"])
        return [loss, logp] + ([grad] if c["grad"] else [])
    x, label = s["logits"].float(), s["label"].long()[:, None]
    most = x.amax(1, keepdim=True)
    e = torch.exp(x - most)
    total = e.sum(1, keepdim=True)
    logp = (x.gather(1, label) - most - torch.log(total))[:, 0]
    w, a = s["weight"], s["advantage"]
    ratio = torch.exp(logp - s["old"])
    free, bounded = ratio * a, ratio.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH) * a
    cut = bounded < free
    d = torch.where(cut, torch.zeros_like(free), -free)
    surrogate, kl = -torch.minimum(free, bounded), torch.zeros_like(w)
    if c["kl"]:
        far = s["ref"] - logp
        kl = torch.exp(far) - far - 1
        d = d + KL * (1 - torch.exp(far))
    sums = [(w * t).sum(dtype=torch.float64) for t in (surrogate, kl, cut.float())]
    loss = torch.stack([sums[0] + KL * sums[1]] + sums).float()
    out = [loss, torch.where(w != 0, logp, torch.zeros_like(logp))]
    if c["grad"]:
        d = (w * d)[:, None]
        e *= -d / total
        e.scatter_add_(1, label, d)
        out.append(s["grad"].copy_(e))
    return out


def _mix(x):
    """32 bits of a 32-bit number, as int64."""
    x = x ^ (x >> 16)
    x = (x * 0x6A09E667) & 0xffffffff
    x = x ^ (x >> 15)
    x = (x * 0xBB67AE85) & 0xffffffff
    return x ^ (x >> 16)


def _random(seed, step, size):
    """16 bits for the first moment and 16 for the second, of each element's number."""
    key = _mix(_mix(seed ^ _mix(step)))  # (of numbers below 2^32)
    bits = _mix((torch.arange(size, device="cuda") + key) & 0xffffffff)
    return (bits & 0xffff).int(), (bits >> 16).int()


def _scaled(x, above):
    """Blocks of x over their power of two, and its byte (255: a value of the block is no finite number)."""
    x = x.view(-1, GROUP)
    exponent = x.abs().amax(1).view(torch.int32) >> 23
    scale = torch.where(exponent == 255, exponent, (exponent - above).clamp(min=1))
    return x * ((254 - scale.clamp(max=253)) << 23).view(torch.float32)[:, None], scale


def _rounded(y, random, lowest):
    """The codes of y >= 0, rounded up with the probability that its distance has; 2^lowest: the smallest normal number, with eight codes below it."""
    small, bias = y < 2.0 ** lowest, (126 + lowest) * 8
    bits = torch.where(small, y + 2.0 ** lowest, y).view(torch.int32)
    return ((bits + (random << 4)) >> 20) - bias - 8 * small.int()


def _to_m(m, random):
    """Sign, four bits of exponent, three of mantissa: 2^-6 to 2^8."""
    y, scale = _scaled(m, 7)
    code = _rounded(y.abs(), random.view(-1, GROUP), -6) | torch.signbit(y).int() << 7
    code = torch.where((scale == 255)[:, None], torch.full_like(code, 127), code)
    return code.to(torch.uint8).view(-1), scale.to(torch.uint8)


def _to_v(v, random):
    """Five bits of exponent, three of mantissa: 2^-14 to 2^16.  What is not zero does not become zero."""
    y, scale = _scaled(v, 15)
    code = _rounded(y, random.view(-1, GROUP), -14)
    code = torch.where(v.view(-1, GROUP) > 0, code.clamp(min=1), code)
    code = torch.where((scale == 255)[:, None], torch.full_like(code, 255), code)
    return code.to(torch.uint8).view(-1), scale.to(torch.uint8)


def _scale_of(byte):
    return torch.where(byte == 255, torch.full_like(byte, 0x7fc00000, dtype=torch.int32), byte.int() << 23).view(torch.float32)


def _from_m(codes, scale):
    return (codes.view(torch.float8_e4m3fn).float().view(-1, GROUP) * _scale_of(scale)[:, None]).view(-1)


def _from_v(codes, scale):
    y = (codes.int() << 20).view(torch.float32) * 2.0 ** 112
    return (y.view(-1, GROUP) * _scale_of(scale)[:, None]).view(-1)


def _adamw8(s):
    if own:
        import paper_2503_01066_amd as A
        A.alch_adamw8_step(s["list"], LR, BETA1, BETA2, EPS, STEP, seed=s["seed"], grad_factor=s["factor"])
    else:
        random_m, random_v = _random(s["seed"], STEP, s["size"])
        g = s["grad"].float() * s["factor"]
        m = _from_m(*s["m"]) * BETA1 + g * (1 - BETA1)
        v = _from_v(*s["v"]) * BETA2 + (g * g) * (1 - BETA2)
        w = s.get("master", s["param"].float())
        change = m / (1 - BETA1 ** STEP) / ((v / (1 - BETA2 ** STEP)).sqrt() + EPS)
        change[:s["plain"]] += DECAY * w[:s["plain"]]
        w -= LR * change
        s["param"].copy_(w)
        for old, new in zip(s["m"] + s["v"], _to_m(m, random_m) + _to_v(v, random_v)):
            old.copy_(new)
    return [s["param"], s["m"], s["v"]] + ([s["master"]] if "master" in s else [])


# ---- what a pass cannot do without, and its outputs in 64 bits ------------------------------------------------------

def work(case):
    E = 2 if case["dtype"] == "bf16" else 4
    if case["op"] in ("pack8", "expand"):
        wide, scales = sum(_widths(case)), 4 * sum(_groups(w) for w in _widths(case))
        if case["op"] == "expand":
            n, lost = case["rows"], case["rows"] // 50 if case["listed"] else 0
            return dict(bytes=(n - lost) * (wide + scales) + n * wide * E + (4 * n if case["listed"] else 0), flops=(n - lost) * wide)
        n = _kept(case)
        return dict(bytes=case["tokens"] + 8 * case["seqs"] + 4 * n + n * (wide * (E + 1) + scales), flops=3 * n * wide)
    if case["op"] == "policy":
        n, V = case["items"], case["vocab"]
        counted = n - int(n * case["masked"])
        return dict(bytes=(counted + (n if case["grad"] else 0)) * V * E + (24 if case["kl"] else 20) * n, flops=counted * V * (7 if case["grad"] else 4))
    n = sum(_lengths(case)[0])
    return dict(bytes=n * (2 * E + 4 + 4 / GROUP + (8 if case["master"] else E)), flops=40 * n)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "pack8":
        at = torch.nonzero(s["mask"])[:, 0]
        scales = []
        for x in s["streams"]:
            parts = x[at].double().abs().split(GROUP, 1)
            scales.append((None, torch.stack([p.max(1).values for p in parts], 1) / 127))
        return None, None, None, scales
    if case["op"] == "expand":
        outs = []
        for (codes, scales), out in zip(s["records"], s["outs"]):
            x = torch.zeros(out.shape, dtype=torch.float64, device="cuda")
            to = torch.arange(case["rows"], device="cuda") if s["rows"] is None else torch.nonzero(s["rows"] >= 0)[:, 0]
            of = to if s["rows"] is None else s["rows"][to].long()
            for k in range(scales.shape[1]):
                x[to, GROUP * k:GROUP * (k + 1)] = codes[of, GROUP * k:GROUP * (k + 1)].double() * scales[of, k].double()[:, None]
            outs.append(x)
        return outs
    if case["op"] == "policy":
        n, loss = case["items"], torch.zeros(4, dtype=torch.float64, device="cuda")
        logps, grads = [], []
        for a in range(0, n, 512):
            b = slice(a, min(a + 512, n))
            every = torch.log_softmax(s["logits"][b].double(), 1)
            at = torch.arange(every.shape[0], device="cuda")
            label = s["label"][b].long()
            logp, w, adv = every[at, label], s["weight"][b].double(), s["advantage"][b].double()
            change = logp - s["old"][b].double()
            ratio = torch.exp(change)
            cut = ((adv > 0) & (ratio > 1 + CLIP_HIGH)) | ((adv < 0) & (ratio < 1 - CLIP_LOW))
            bound = torch.where(adv > 0, torch.full_like(adv, 1 + CLIP_HIGH), torch.full_like(adv, 1 - CLIP_LOW))
            surrogate = -torch.where(cut, bound, ratio) * adv
            d = torch.where(cut, torch.zeros_like(adv), -ratio * adv)
            kl = torch.zeros_like(adv)
            if case["kl"]:
                gap = s["ref"][b].double() - logp
                kl = torch.expm1(gap) - gap
                d -= KL * torch.expm1(gap)
            loss += torch.stack([(w * (surrogate + KL * kl)).sum(), (w * surrogate).sum(), (w * kl).sum(), (w * cut).sum()])
            logps.append(torch.where(w > 0, logp, torch.zeros_like(logp)))
            if case["grad"]:
                x = torch.exp(every) * -(w * d)[:, None]
                x[at, label] += w * d
                grads.append(x)
        return [loss, torch.cat(logps)] + ([torch.cat(grads)] if case["grad"] else [])
    power = lambda byte: torch.pow(torch.full((1,), 2.0, dtype=torch.float64, device="cuda"), byte.double() - 127).repeat_interleave(GROUP)
    g = s["grad"].double() * float(s["factor"])
    v_code = s["v"][0].long()
    exponent, mantissa = v_code // 8, (v_code % 8).double() / 8
    v = torch.where(exponent > 0, (1 + mantissa) * torch.exp2((exponent - 15).double()), mantissa * 2.0 ** -14) * power(s["v"][1])
    m = s["m"][0].view(torch.float8_e4m3fn).double() * power(s["m"][1])
    m, v = BETA1 * m + (1 - BETA1) * g, BETA2 * v + (1 - BETA2) * g.square()
    w = s.get("master", s["param"]).double()
    decay = torch.zeros(s["size"], dtype=torch.float64, device="cuda")
    decay[:s["plain"]] = DECAY
    w = w - LR * (m / (1 - BETA1 ** STEP) / (torch.sqrt(v / (1 - BETA2 ** STEP)) + EPS) + decay * w)
    return [w, (None, None), (None, None)] + ([w] if "master" in s else [])
