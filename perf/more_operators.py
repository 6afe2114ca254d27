"""What a training step has at its two ends and between its blocks, as the library is timed on it, with plain forms.

Three operators, each case one pass of a training or inference program:

* ``embed``: a model's input, the scaled sum of one table row for each of a token's or node's ids (a vocabulary; a
  node's categorical features and its degree encodings), forward, or forward and the table's gradient;
* ``dropout``: dropout of a block's output from a counter-based generator, with the residual's addition, forward, or
  forward and backward (no mask is kept, the backward draws the same numbers again);
* ``loss``: softmax cross entropy over many classes straight from the last features and the class weights, forward, or
  forward and the gradients of both.  Rows whose label is no class (unlabelled nodes, prompt tokens) have none.

Values are made on the GPU from the seed.
"""

import math

import torch

own = False  # True: the framework's calls; False: the plain forms below

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
IT = {"i32": torch.int32, "i64": torch.int64}


def listed():
    return [
        # the next token of 16 sequences being generated: latency
        dict(name="embed_few", op="embed", mode="fwd", dtype="bf16", ids="i64", rows=16, fields=1, table=128_000,
             width=2048),
        # a training step's tokens, four sequences of 4,096
        dict(name="embed_tokens_step", op="embed", mode="step", dtype="bf16", ids="i64", rows=16_384, fields=1,
             table=128_000, width=2048),
        # a million nodes: a node type and the encodings of the in- and out-degree
        dict(name="embed_nodes_step", op="embed", mode="step", dtype="bf16", ids="i32", rows=1_000_000, fields=3,
             table=1_500, width=256),
        # the atoms of 4,000 molecules, nine categorical features each, in single precision
        dict(name="embed_atoms_step", op="embed", mode="step", dtype="f32", ids="i64", rows=100_000, fields=9,
             table=173, width=256),
        # dropout of a handful of rows: latency
        dict(name="dropout_few", op="dropout", mode="fwd", dtype="f32", rows=7, width=512, p=0.1, add=True),
        # a training step's block output at 100,000 nodes of 512 features, with the residual
        dict(name="dropout_100k_step", op="dropout", mode="step", dtype="bf16", rows=100_000, width=512, p=0.1,
             add=True),
        # the input's dropout at a million nodes of 256 features
        dict(name="dropout_1m_step", op="dropout", mode="step", dtype="bf16", rows=1_000_000, width=256, p=0.5,
             add=False),
        # a few nodes of a small graph over 40 classes: latency
        dict(name="loss_few", op="loss", mode="step", dtype="f32", ids="i64", rows=33, classes=40, width=64,
             labelled=1.0),
        # node classification: 200,000 nodes, three in ten of them labelled, 172 classes
        dict(name="loss_nodes_step", op="loss", mode="step", dtype="bf16", ids="i64", rows=200_000, classes=172,
             width=256, labelled=0.3),
        # scoring one token of each of 16 sequences over a vocabulary: the weights are read once
        dict(name="loss_score_few", op="loss", mode="fwd", dtype="bf16", ids="i64", rows=16, classes=128_000,
             width=2048, labelled=1.0),
        # a training step over a vocabulary, the prompts' tokens without a label
        dict(name="loss_vocab_step", op="loss", mode="step", dtype="bf16", ids="i64", rows=8192, classes=128_000,
             width=2048, labelled=0.85),
        # the same in single precision over a smaller vocabulary
        dict(name="loss_f32_step", op="loss", mode="step", dtype="f32", ids="i32", rows=2048, classes=32_000,
             width=512, labelled=1.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["embed", "embed", "dropout", "loss", "loss", "loss"])
    dtype, mode = rng.choice(["bf16", "bf16", "f32"]), rng.choice(["fwd", "step", "step"])
    size = 2 if dtype == "bf16" else 4
    while True:
        width = rng.choice([_log(rng, 1, 40), 64 * rng.randint(1, 16), 64 * rng.randint(1, 32), _log(rng, 33, 4200)])
        if op == "embed":
            c = dict(op=op, mode=mode, dtype=dtype, ids=rng.choice(["i32", "i64"]), rows=_log(rng, 1, 1_000_000),
                     fields=rng.choice([1, 1, 1, 2, 3, rng.randint(4, 12)]), table=_log(rng, 1, 300_000), width=width)
            if c["rows"] * width * size > 5.2e8 or c["table"] * width * size > 5.2e8:
                continue
            if c["rows"] * c["fields"] * width > 7.5e8 or c["fields"] > c["table"]:
                continue
            return c
        if op == "dropout":
            c = dict(op=op, mode=mode, dtype=dtype, rows=_log(rng, 1, 1_000_000), width=width,
                     p=rng.choice([0.1, 0.5, round(rng.uniform(0.0, 0.9), 3)]), add=rng.random() < 0.5)
            if c["rows"] * width * size > 5.2e8:
                continue
            return c
        c = dict(op=op, mode=mode, dtype=dtype, ids=rng.choice(["i32", "i64"]), rows=_log(rng, 1, 400_000),
                 classes=_log(rng, 2, 260_000), width=width, labelled=rng.choice([1.0, 1.0, 0.85, 0.3]))
        most = 2.1e12 if dtype == "bf16" else 1.4e11
        if c["rows"] * c["classes"] > 1.05e9 or c["rows"] * c["classes"] * max(width, 64) > most:
            continue
        if max(c["rows"], c["classes"]) * width * size > 5.3e8:
            continue
        if mode == "step" and c["rows"] * c["labelled"] < 8:  # a mean over nothing
            continue
        return c


# ---------------------------------------------------------------------------------------------- inputs

def _normal(g, dtype, *shape):
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def _ids(g, shape, most):
    """Ids as tokens, degrees and categories come: a few frequent ones and a long tail."""
    u = torch.rand(shape, generator=g, device="cuda", dtype=torch.float64)
    return (torch.exp(u * math.log(most + 1.0)) - 1.0).long().clamp_(0, most - 1)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    s, dt, w, n = {"case": case}, DT[case["dtype"]], case["width"], case["rows"]
    if case["op"] == "embed":
        s["table"] = _normal(g, dt, case["table"], w)
        f, r = case["fields"], case["table"]
        # each field has its own share of the table; one id in 50 is unknown and adds nothing
        at = [r * k // f for k in range(f + 1)]
        ids = torch.stack([at[k] + _ids(g, (n,), at[k + 1] - at[k]) for k in range(f)], 1)
        ids[torch.rand(n, f, generator=g, device="cuda") < 0.02] = -1
        s["ids"] = ids.to(IT[case["ids"]])
        s["scale"] = math.sqrt(w) if f == 1 else 1.0
        s["dout"] = _normal(g, dt, n, w)
        return s
    if case["op"] == "dropout":
        s["x"], s["dy"] = _normal(g, dt, n, w), _normal(g, dt, n, w)
        s["add"] = _normal(g, dt, n, w) if case["add"] else None
        # seed and offset of the generator, on the GPU
        s["rng"] = torch.randint(-2 ** 62, 2 ** 62, (2,), generator=g, device="cuda")
        return s
    v = case["classes"]
    s["x"] = _normal(g, dt, n, w)
    s["w"] = (torch.randn(v, w, generator=g, device="cuda") * (2.0 / math.sqrt(w))).to(dt)
    labels = _ids(g, (n,), v)
    labels[torch.rand(n, generator=g, device="cuda") >= case["labelled"]] = -100
    s["labels"] = labels.to(IT[case["ids"]])
    # the upstream gradient of a mean over the labelled rows
    s["dloss"] = torch.full((n,), 1.0, device="cuda") / (labels >= 0).sum().clamp(min=1)
    return s


# ------------------------------------------------------------------------------------------- the calls

def run(s):
    case = s["case"]
    step = case["mode"] == "step"
    if not own:
        return {"embed": _plain_embed, "dropout": _plain_dropout, "loss": _plain_loss}[case["op"]](s)
    from paper_2407_14106_amd import gt
    if case["op"] == "embed":
        out = gt.embed_fwd(s["table"], s["ids"], scale=s["scale"])
        return (out, gt.embed_bwd(s["ids"], s["dout"], case["table"], scale=s["scale"])) if step else out
    if case["op"] == "dropout":
        y = gt.dropout(s["x"], case["p"], s["rng"], add=s["add"])
        return (y, gt.dropout(s["dy"], case["p"], s["rng"])) if step else y
    loss, lse = gt.class_loss_fwd(s["x"], s["w"], s["labels"])
    if not step:
        return loss, lse
    return (loss, lse) + gt.class_loss_bwd(s["x"], s["w"], s["labels"], lse, s["dloss"])


# ------------------------------------------------------------------------------------- the plain forms

def _plain_embed(s):
    case, dt = s["case"], DT[s["case"]["dtype"]]
    ids, out = s["ids"].long(), 0.0
    for f in range(case["fields"]):
        there = (ids[:, f] >= 0) & (ids[:, f] < case["table"])
        out = out + s["table"][torch.where(there, ids[:, f], 0)].float() * there[:, None]
    out = (out * s["scale"]).to(dt)
    if case["mode"] == "fwd":
        return out
    # the ids sorted, an id's sum is the difference of two running sums; these are long: 64 bits
    r, w = case["table"], case["width"]
    key, order = torch.sort(torch.where((ids >= 0) & (ids < r), ids, r).reshape(-1), stable=True)
    ends = torch.searchsorted(key, torch.arange(r, device="cuda"), right=True)
    starts = torch.searchsorted(key, torch.arange(r, device="cuda"))
    rows = order // case["fields"]
    grad = torch.empty(r, w, dtype=dt, device="cuda")
    some = max(1, int(3e8 // rows.numel()))  # features at a time
    for c in range(0, w, some):
        run = s["dout"][:, c:c + some].t().contiguous()[:, rows].double().cumsum_(1)
        run = torch.nn.functional.pad(run, (1, 0))
        grad[:, c:c + some] = ((run[:, ends] - run[:, starts]) * s["scale"]).t().to(dt)
    return out, grad


def _words(rng, n):
    """The generator's n 32-bit words: Philox4x32-10 (Salmon et al., SC 2011), four for each counter."""
    low = 0xFFFFFFFF
    c = torch.arange((n + 3) // 4, device="cuda") + rng[1]
    x = [c & low, (c >> 32) & low, torch.zeros_like(c), torch.zeros_like(c)]
    k = [rng[0] & low, (rng[0] >> 32) & low]
    for _ in range(10):
        a, b = x[0] * 0xD2511F53, x[2] * 0xCD9E8D57
        x = [((b >> 32) & low) ^ x[1] ^ k[0], b & low, ((a >> 32) & low) ^ x[3] ^ k[1], a & low]
        k = [(k[0] + 0x9E3779B9) & low, (k[1] + 0xBB67AE85) & low]
    return torch.stack(x, 1).view(-1)[:n]


def _plain_dropout(s):
    case, dt = s["case"], DT[s["case"]["dtype"]]
    keep = (_words(s["rng"], s["x"].numel()) >= round(case["p"] * 2.0 ** 32)).view(s["x"].shape)
    up = 1.0 / (1.0 - case["p"])
    y = torch.where(keep, s["x"].float() * up, 0.0)
    if case["add"]:
        y = y + s["add"].float()
    y = y.to(dt)
    return y if case["mode"] == "fwd" else (y, torch.where(keep, s["dy"].float() * up, 0.0).to(dt))


def _plain_loss(s):
    case, dt = s["case"], DT[s["case"]["dtype"]]
    rows = torch.nonzero((s["labels"] >= 0) & (s["labels"] < case["classes"]))[:, 0]
    y = s["labels"].long()[rows]
    x, w = s["x"].float()[rows], s["w"].float()
    p = torch.matmul(x, w.t())
    at = torch.arange(rows.numel(), device="cuda")
    top = p.amax(1, keepdim=True)
    hit = p[at, y]
    lse_r = (top + torch.log(torch.exp(p - top).sum(1, keepdim=True)))[:, 0]
    loss, lse = torch.zeros(case["rows"], device="cuda"), torch.zeros(case["rows"], device="cuda")
    loss[rows], lse[rows] = lse_r - hit, lse_r
    if case["mode"] == "fwd":
        return loss, lse
    p = torch.exp(p - lse_r[:, None])
    p[at, y] -= 1.0
    p *= s["dloss"][rows, None]
    dx = torch.zeros(case["rows"], case["width"], device="cuda")
    dx[rows] = torch.matmul(p, w)
    return loss, lse, dx.to(dt), torch.matmul(p.t(), x).to(dt)


# ------------------------------------------------------------------------------------ work and 64 bits

def work(case):
    n, w, b, step = case["rows"], case["width"], 2 if case["dtype"] == "bf16" else 4, case["mode"] == "step"
    ib = 4 if case.get("ids") == "i32" else 8
    if case["op"] == "embed":
        pairs, r = n * case["fields"], case["table"]
        fwd = ib * pairs + b * w * (n + min(r, pairs))
        return {"bytes": fwd + step * (ib * pairs + b * w * (n + r)), "flops": pairs * w * (2 if step else 1)}
    if case["op"] == "dropout":
        return {"bytes": b * n * w * (2 + case["add"] + 2 * step), "flops": 2 * n * w * (2 if step else 1)}
    v, m = case["classes"], max(1, round(n * case["labelled"]))
    # the logits are not kept, so the backward forms them again
    return {"bytes": (b * w * (m + v) + ib * n) * (2 if step else 1) + 8 * n + step * (b * w * (n + v) + 8 * n),
            "flops": 2 * m * v * w * (4 if step else 1)}


def exact(case, seed):
    s = prepare(case, seed)
    return {"embed": _exact_embed, "dropout": _exact_dropout, "loss": _exact_loss}[case["op"]](s, case)


def _exact_embed(s, case):
    r, w = case["table"], case["width"]
    more = torch.cat([s["table"].double(), torch.zeros(1, w, dtype=torch.float64, device="cuda")])
    ids = s["ids"].long()
    ids = torch.where((ids < 0) | (ids >= r), r, ids)
    out = sum(more[ids[:, f]] for f in range(case["fields"])) * s["scale"]
    if case["mode"] == "fwd":
        return out
    grad = torch.zeros(r + 1, w, dtype=torch.float64, device="cuda")
    for f in range(case["fields"]):
        grad.index_add_(0, ids[:, f], s["dout"].double())
    return out, grad[:-1] * s["scale"]


def _exact_dropout(s, case):
    n = s["x"].numel()
    seed, offset = (int(v) % 2 ** 64 for v in s["rng"].tolist())

    def times(a, b):  # (high, low) words of the product, by 16-bit limbs
        a0, a1, b0, b1 = a & 0xFFFF, a >> 16, b & 0xFFFF, b >> 16
        mid = a1 * b0 + (a0 * b0 >> 16)
        mid2 = a0 * b1 + (mid & 0xFFFF)
        return a1 * b1 + (mid >> 16) + (mid2 >> 16), (mid2 & 0xFFFF) << 16 | a0 * b0 & 0xFFFF

    keep = torch.empty(n, dtype=torch.bool, device="cuda")
    part = 1 << 24  # counters at a time
    for c in range(0, (n + 3) // 4, part):
        i = torch.arange(c, min(c + part, (n + 3) // 4), device="cuda")
        low = i + (offset & 0xFFFFFFFF)
        r, l = low & 0xFFFFFFFF, ((low >> 32) + (offset >> 32)) & 0xFFFFFFFF
        r2 = l2 = torch.zeros_like(r)
        for t in range(10):
            k0 = ((seed & 0xFFFFFFFF) + t * 0x9E3779B9) & 0xFFFFFFFF
            k1 = ((seed >> 32) + t * 0xBB67AE85) & 0xFFFFFFFF
            (h0, m0), (h1, m1) = times(r, 0xD2511F53), times(r2, 0xCD9E8D57)
            r, l, r2, l2 = h1 ^ l ^ k0, m1, h0 ^ l2 ^ k1, m0
        for j, word in enumerate((r, l, r2, l2)):
            room = keep[4 * c + j:4 * (c + i.numel()):4]
            room.copy_((word >= round(case["p"] * 2 ** 32))[:room.numel()])
    keep = keep.view(s["x"].shape)
    zero = torch.zeros((), dtype=torch.float64, device="cuda")
    y = torch.where(keep, s["x"].double() / (1.0 - case["p"]), zero)
    if case["add"]:
        y = y + s["add"].double()
    return y if case["mode"] == "fwd" else (y, torch.where(keep, s["dy"].double() / (1.0 - case["p"]), zero))


def _exact_loss(s, case):
    f64 = dict(dtype=torch.float64, device="cuda")
    n, v, w = case["rows"], case["classes"], case["width"]
    weight, x = s["w"].double(), s["x"].double()
    turned = weight.t().contiguous()
    loss, lse, dx, dw = torch.zeros(n, **f64), torch.zeros(n, **f64), torch.zeros(n, w, **f64), torch.zeros(v, w, **f64)
    some = max(1, int(3e8 // v))  # rows at a time
    for a in range(0, n, some):
        y = s["labels"][a:a + some].long()
        has = (y >= 0) & (y < v)
        y = torch.where(has, y, 0)
        z = torch.mm(x[a:a + some], turned)
        lse_r = torch.logsumexp(z, 1)
        lse[a:a + some] = torch.where(has, lse_r, 0.0)
        loss[a:a + some] = torch.where(has, lse_r - z.gather(1, y[:, None])[:, 0], 0.0)
        if case["mode"] == "step":
            z = torch.exp(z - lse_r[:, None]).scatter_add_(1, y[:, None], torch.full_like(z[:, :1], -1.0))
            z *= torch.where(has, s["dloss"][a:a + some].double(), 0.0)[:, None]
            dx[a:a + some] = torch.mm(z, weight)
            dw += torch.mm(z.t().contiguous(), x[a:a + some])
    return (loss, lse, dx, dw) if case["mode"] == "step" else (loss, lse)
