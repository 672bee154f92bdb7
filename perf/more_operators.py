"""The measured work of the operators around an encoder's blocks: what training
a text encoder on its own tokens needs besides attention.

Token ids become rows of a table and the table's gradient is summed by token;
every block's output is added to the residual stream between a norm of its own
and the norm of the next block; and the last rows are scored against a large
table of classes (the words of a vocabulary, or the rows of other documents)
under a softmax cross entropy.  Training runs the backward passes too.  Each
case below is one such call (a training case: the forward call and its backward
call).  Values come from the seed.
"""
import math

import torch

own = False

DEV = "cuda"
EPS = 1e-5
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32,
          "int32": torch.int32, "int64": torch.int64}


def listed():
    return [
        # the tokens of one short text on its way to the search: pure latency
        dict(name="embed_text", op="embed", tokens=23, vocab=50_000, width=768, table="bf16", dtype="bf16",
             scaled=True, mask=0.0, pad=0.0, ids="int64"),
        # a corpus batch, from the 32-bit table that an optimiser keeps
        dict(name="embed_corpus", op="embed", tokens=200_003, vocab=64_000, width=1024, table="fp32", dtype="bf16",
             scaled=True, mask=0.0, pad=0.0, ids="int64"),
        # a masked training batch: words as often as in text, one in eight the mask
        dict(name="embed_train", op="embed_train", tokens=131_000, vocab=64_000, width=768, table="bf16",
             dtype="bf16", scaled=True, mask=0.12, pad=0.0, ids="int64"),
        # few tokens, padded, against a large table of an odd width
        dict(name="embed_odd", op="embed_train", tokens=9_001, vocab=100_003, width=301, table="fp32", dtype="fp32",
             scaled=False, mask=0.0, pad=0.1, ids="int32"),
        # the rows of one short text between two blocks: pure latency
        dict(name="step_text", op="step", rows=23, width=768, dtype="bf16", weights="bf16", rms=False, pre=True,
             post=True, bias=True, gate="column", alpha=1.0),
        # a corpus batch, inference
        dict(name="step_corpus", op="step", rows=200_003, width=1024, dtype="bf16", weights="fp32", rms=True, pre=True,
             post=True, bias=False, gate="column", alpha=1.0),
        # a training batch between two blocks: both outputs, and every gradient
        dict(name="step_train", op="step_train", rows=100_003, width=768, dtype="bf16", weights="bf16", rms=False,
             pre=True, post=True, bias=True, gate="column", alpha=1.0),
        # an odd width in 32 bits, a gate for every element, the stream scaled up
        dict(name="step_odd", op="step_train", rows=20_011, width=1001, dtype="fp32", weights="fp32", rms=True,
             pre=True, post=True, bias=False, gate="row", alpha=1.25),
        # the masked words of one short text: the table is all the work
        dict(name="loss_text", op="loss", rows=5, classes=50_000, width=768, dtype="bf16", live=1.0, bias=True,
             scale=1.0, weighted=False, ids="int64"),
        # a masked training batch: one token in seven has a target
        dict(name="loss_masked", op="loss_train", rows=32_768, classes=50_001, width=768, dtype="bf16", live=0.15,
             bias=True, scale=1.0, weighted=False, ids="int64"),
        # every token has a target, a large vocabulary
        dict(name="loss_large", op="loss_train", rows=8_192, classes=131_072, width=1024, dtype="bf16", live=1.0,
             bias=False, scale=1.0, weighted=False, ids="int64"),
        # unit rows against the unit rows of their duplicates and of others, at a temperature of 0.05
        dict(name="loss_pairs", op="loss_train", rows=4_099, classes=32_800, width=256, dtype="fp16", live=1.0,
             bias=False, scale=20.0, weighted=False, ids="int32"),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["embed", "embed_train", "embed_train", "step", "step_train", "step_train", "loss", "loss_train",
                     "loss_train", "loss_train"])
    if op in ("embed", "embed_train"):
        width = rng.choice([64, 96, 256, 384, 512, 768, 1024, 2048, _spread(rng, 1, 4096)])
        vocab = min(_spread(rng, 2, 262_144), 100_000_000 // width)
        return dict(op=op, tokens=min(_spread(rng, 1, 262_144), 100_000_000 // width), vocab=vocab, width=width,
                    table=rng.choice(["bf16", "fp16", "fp32"]), dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]),
                    scaled=rng.random() < 0.5, mask=rng.choice([0.0, 0.0, 0.12, 0.5]), pad=rng.choice([0.0, 0.0, 0.2]),
                    ids=rng.choice(["int32", "int64"]))
    if op in ("step", "step_train"):
        width = rng.choice([64, 96, 256, 384, 512, 768, 1024, 2048, _spread(rng, 1, 4096)])
        dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
        pre = rng.random() < 0.8
        return dict(op=op, rows=_spread(rng, 1, min(200_000, 50_000_000 // width)), width=width, dtype=dtype,
                    weights=rng.choice([dtype, "fp32"]), rms=rng.random() < 0.5, pre=pre,
                    post=not pre or rng.random() < 0.6, bias=rng.random() < 0.6,
                    gate=rng.choice(["none", "column", "column", "row"]), alpha=rng.choice([1.0, 1.0, 0.5, 1.6]))
    width = rng.choice([64, 128, 256, 384, 512, 768, 1024, 2048, 8 * _spread(rng, 1, 256)])
    classes = _spread(rng, 2, 131_072)
    most = 1.05e12 / (classes * width)
    live = rng.choice([1.0, 1.0, 0.5, 0.15])
    return dict(op=op, rows=int(max(1, min(_spread(rng, 1, 16_384), most / live, 1.1e9 / classes))), classes=classes,
                width=width, dtype=rng.choice(["bf16", "bf16", "fp16"]), live=live, bias=rng.random() < 0.5,
                scale=rng.choice([1.0, 1.0, 20.0]), weighted=rng.random() < 0.3, ids=rng.choice(["int32", "int64"]))


def _size(name):
    return torch.empty(0, dtype=DTYPES[name]).element_size()


def _live_rows(case):
    """The rows that have a target: a fixed number, spread by the seed."""
    return max(1, int(round(case["rows"] * case["live"])))


def work(case):
    if case["op"] in ("embed", "embed_train"):
        n, w, v = case["tokens"], case["width"], case["vocab"]
        real = n - int(n * case["pad"])
        # the different words among the tokens, on average
        often = torch.log1p(1 / torch.arange(1, v + 1, dtype=torch.float64)) / math.log(v + 1) * (1 - case["mask"])
        words = float(-torch.expm1(real * torch.log1p(-often.clamp(max=1 - 1e-12))).sum())
        out = {"bytes": int(n * _size(case["ids"]) + words * w * _size(case["table"]) + n * w * _size(case["dtype"])),
               "flops": n * w}
        if case["op"] == "embed_train":                    # the gradient: 32 bits, every row of the table
            out["bytes"] += n * _size(case["ids"]) + real * w * _size(case["dtype"]) + v * w * 4
            out["flops"] += n * w
        return out
    if case["op"] in ("step", "step_train"):
        n, w = case["rows"], case["width"]
        gate = case["gate"] == "row"
        vectors = case["pre"] * (1 + case["bias"]) + case["post"] * (1 + case["bias"]) + (case["gate"] == "column")
        out = {"bytes": (3 + case["pre"] + gate) * n * w * _size(case["dtype"]) + vectors * w * _size(case["weights"]),
               "flops": 12 * n * w}
        if case["op"] == "step_train":
            # y and the gradient of the stream (of x, and h), a gate of rows; dh, dy, the gate's
            out["bytes"] += (4 + 2 * case["pre"] + 2 * gate) * n * w * _size(case["dtype"])
            out["bytes"] += 2 * vectors * w * _size(case["weights"])
            out["flops"] += 36 * n * w
        return out
    n, v, d, size = _live_rows(case), case["classes"], case["width"], _size(case["dtype"])
    out = {"bytes": (n + v) * d * size + (4 * v if case["bias"] else 0) + case["rows"] * (8 + _size(case["ids"])),
           "flops": 2 * n * v * d}
    if case["op"] == "loss_train":
        # the backward pass: both inputs again, both gradients; the scores anew and a product for each gradient
        out["bytes"] += (n + v) * d * size + (case["rows"] + v) * d * size + (8 * v if case["bias"] else 0) + 12 * case["rows"]
        out["flops"] += 6 * n * v * d
    return out


# ---------------------------------------------------------------------------
# what a program has in hand
def prepare(case, seed):
    g = torch.Generator(DEV).manual_seed(seed)

    def randn(*shape):
        return torch.randn(*shape, generator=g, device=DEV)

    def rand(*shape):
        return torch.rand(*shape, generator=g, device=DEV)

    st = {"case": case}
    if case["op"] in ("embed", "embed_train"):
        n, v, w = case["tokens"], case["vocab"], case["width"]
        st["table"] = (randn(v, w) * w ** -0.5).to(DTYPES[case["table"]])
        # words as often as in text: the k-th most frequent 1/k as often as the first
        ids = torch.exp(rand(n).double() * math.log(v + 1)).long().sub_(1).clamp_(0, v - 1)
        if case["mask"]:
            ids = torch.where(rand(n) < case["mask"], min(3, v - 1), ids)
        if case["pad"]:
            ids[torch.randperm(n, generator=g, device=DEV)[:int(n * case["pad"])]] = -1
        st["ids"] = ids.to(DTYPES[case["ids"]])
        st["scale"] = w ** 0.5 if case["scaled"] else 1.0
        if case["op"] == "embed_train":
            st["dout"] = randn(n, w).to(DTYPES[case["dtype"]])
        return st
    if case["op"] in ("step", "step_train"):
        n, w = case["rows"], case["width"]
        dtype, wd = DTYPES[case["dtype"]], DTYPES[case["weights"]]
        # the stream: channels of unequal spread around their own means; a block's output is smaller
        st["h"] = (randn(n, w) * torch.exp(0.5 * randn(w)) + 0.3 * randn(w)).to(dtype)
        st["y"] = (0.4 * randn(n, w) * torch.exp(0.3 * randn(w)) + 0.1 * randn(w)).to(dtype)
        st["weight"] = (1 + 0.1 * randn(w)).to(wd) if case["pre"] else None
        st["bias"] = (0.1 * randn(w)).to(wd) if case["pre"] and case["bias"] else None
        st["post_weight"] = (1 + 0.1 * randn(w)).to(wd) if case["post"] else None
        st["post_bias"] = (0.1 * randn(w)).to(wd) if case["post"] and case["bias"] else None
        st["gate"] = {"none": lambda: None, "column": lambda: (0.5 + 0.2 * randn(w)).to(wd),
                      "row": lambda: torch.sigmoid(randn(n, w)).to(dtype)}[case["gate"]]()
        if case["op"] == "step_train":
            st["dx"] = randn(n, w).to(dtype) if case["pre"] else None
            st["dstream"] = randn(n, w).to(dtype)
        return st
    n, v, d, dtype = case["rows"], case["classes"], case["width"], DTYPES[case["dtype"]]
    live = torch.randperm(n, generator=g, device=DEV)[:_live_rows(case)]
    if case["scale"] == 1.0:
        # a table of words around a common direction; rows that point to their word more or less clearly
        table = (randn(v, d) + 0.5 * randn(d)) * 2.5 * d ** -0.5
        word = torch.exp(rand(n).double() * math.log(v + 1)).long().sub_(1).clamp_(0, v - 1)
        h = randn(n, d) + 2.0 * rand(n, 1) * table[word] / 2.5
    else:
        # unit rows, each one's duplicate among the classes, and a few more rows about the same thing
        topic = torch.randint(max(1, v // 4), (v,), generator=g, device=DEV)
        table = randn(max(1, v // 4), d)[topic] + 0.5 * randn(v, d)
        table = table / table.square().sum(1, keepdim=True).sqrt()
        word = torch.randperm(v, generator=g, device=DEV)[:n] if n <= v else torch.randint(v, (n,), generator=g, device=DEV)
        h = table[word] + (0.3 + rand(n, 1)) * randn(n, d) * d ** -0.5
        h = h / h.square().sum(1, keepdim=True).sqrt()
    st["h"], st["weight"] = h.to(dtype), table.to(dtype)
    st["bias"] = 0.5 * randn(v) if case["bias"] else None
    targets = torch.full((n,), -1, dtype=torch.int64, device=DEV)
    targets[live] = word[live]
    st["targets"] = targets.to(DTYPES[case["ids"]])
    # the mean over the rows with a target; fp16 training scales its loss up
    up = 4096.0 if case["dtype"] == "fp16" else 1.0
    st["dloss"] = (0.5 + rand(n) if case["weighted"] else torch.ones(n, device=DEV)) * (up / _live_rows(case))
    return st


# ---------------------------------------------------------------------------
# one pass
def run(st):
    op = st["case"]["op"]
    if op in ("embed", "embed_train"):
        return _own_embed(st) if own else _plain_embed(st)
    if op in ("step", "step_train"):
        return _own_step(st) if own else _plain_step(st)
    return _own_loss(st) if own else _plain_loss(st)


def _own_embed(st):
    import paper_2608_03199_gb300 as sieve
    c = st["case"]
    out = sieve.embed(st["ids"], st["table"], scale=st["scale"], dtype=DTYPES[c["dtype"]])
    if c["op"] == "embed":
        return {"out": out}
    return {"out": out, "dtable": sieve.embed_backward(st["dout"], st["ids"], c["vocab"], scale=st["scale"])}


def _own_step(st):
    import paper_2608_03199_gb300 as sieve
    c = st["case"]
    kw = dict(weight=st["weight"], bias=st["bias"], post_weight=st["post_weight"], post_bias=st["post_bias"],
              gate=st["gate"], alpha=c["alpha"], rms=c["rms"])
    stream, x, stats = sieve.residual_norm(st["h"], st["y"], eps=EPS, **kw)
    res = {"stream": stream, "x": x}
    if c["op"] == "step_train":
        grads = sieve.residual_norm_backward(st["dstream"], st["dx"], st["h"], st["y"], stats, **kw)
        res.update(zip(("dh", "dy", "dweight", "dbias", "dpost_weight", "dpost_bias", "dgate"), grads))
    return {k: t for k, t in res.items() if t is not None}


def _own_loss(st):
    import paper_2608_03199_gb300 as sieve
    c = st["case"]
    loss, lse = sieve.cross_entropy(st["h"], st["weight"], st["targets"], bias=st["bias"], scale=c["scale"])
    res = {"loss": loss, "lse": lse}
    if c["op"] == "loss_train":
        dh, dweight, dbias = sieve.cross_entropy_backward(st["dloss"], st["h"], st["weight"], st["targets"], loss,
                                                          lse, bias=st["bias"], scale=c["scale"])
        res.update(dh=dh, dweight=dweight)
        if c["bias"]:
            res["dbias"] = dbias
    return res


def _plain_embed(st):
    c, ids = st["case"], st["ids"].long()
    real = (ids >= 0) & (ids < c["vocab"])
    out = torch.where(real[:, None], st["table"][torch.where(real, ids, 0)].float() * st["scale"], 0.0)
    out = out.to(DTYPES[c["dtype"]])
    if c["op"] == "embed":
        return {"out": out}
    d = torch.where(real[:, None], st["dout"].float() * st["scale"], 0.0)
    # (sums of thousands of rows: 64 bits)
    dtable = torch.zeros(c["vocab"], c["width"], device=DEV, dtype=torch.float64).index_add_(
        0, torch.where(real, ids, 0), d.double())
    return {"out": out, "dtable": dtable.float()}


def _plain_norm(x, weight, bias, rms):
    """Output, normalised rows and their factor."""
    centred = x if rms else x - x.mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(centred.square().mean(1, keepdim=True) + EPS)
    unit = centred * rstd
    out = unit * weight.float()
    return (out if bias is None else out + bias.float()), unit, rstd


def _plain_norm_grad(dout, weight, unit, rstd, rms):
    d = dout * weight.float()
    back = d - unit * (d * unit).mean(1, keepdim=True)
    return rstd * (back if rms else back - d.mean(1, keepdim=True))


def _plain_step(st):
    c, dtype, wd = st["case"], DTYPES[st["case"]["dtype"]], DTYPES[st["case"]["weights"]]
    rms, gate = c["rms"], 1.0 if st["gate"] is None else st["gate"].float()
    u = y = st["y"].float()
    if c["post"]:
        u, unit1, rstd1 = _plain_norm(y, st["post_weight"], st["post_bias"], rms)
    stream = c["alpha"] * st["h"].float() + gate * u
    res = {"stream": stream.to(dtype)}
    if c["pre"]:
        x, unit2, rstd2 = _plain_norm(stream, st["weight"], st["bias"], rms)
        res["x"] = x.to(dtype)
    if c["op"] == "step":
        return res
    g = st["dstream"].float()
    if c["pre"]:
        dx = st["dx"].float()
        g = g + _plain_norm_grad(dx, st["weight"], unit2, rstd2, rms)
    res["dh"] = (c["alpha"] * g).to(dtype)
    du = g * gate
    res["dy"] = (_plain_norm_grad(du, st["post_weight"], unit1, rstd1, rms) if c["post"] else du).to(dtype)
    if c["pre"]:
        res["dweight"] = (dx * unit2).sum(0).to(wd)
        if c["bias"]:
            res["dbias"] = dx.sum(0).to(wd)
    if c["post"]:
        res["dpost_weight"] = (du * unit1).sum(0).to(wd)
        if c["bias"]:
            res["dpost_bias"] = du.sum(0).to(wd)
    if c["gate"] != "none":
        res["dgate"] = (g * u).sum(0).to(wd) if c["gate"] == "column" else (g * u).to(dtype)
    return res


def _plain_loss(st):
    c, dtype, t = st["case"], st["h"].dtype, st["targets"].long()
    n, v = c["rows"], c["classes"]
    at = ((t >= 0) & (t < v)).nonzero()[:, 0]
    x, w, t = st["h"][at].float(), st["weight"].float(), t[at][:, None]
    z = x @ w.t()
    z *= c["scale"]
    if c["bias"]:
        z += st["bias"]
    top = z.amax(1, keepdim=True)
    hit = z.gather(1, t)
    e = torch.exp_(z.sub_(top))
    total = e.sum(1, keepdim=True)
    lse = top + torch.log(total)
    res = {"loss": torch.zeros(n, device=DEV).index_copy_(0, at, (lse - hit)[:, 0]),
           "lse": torch.zeros(n, device=DEV).index_copy_(0, at, lse[:, 0])}
    if c["op"] == "loss":
        return res
    dz = e.mul_(1 / total)
    dz.scatter_add_(1, t, torch.full_like(hit, -1.0))
    dz *= st["dloss"][at][:, None]
    dh = torch.zeros(n, c["width"], device=DEV).index_copy_(0, at, c["scale"] * (dz @ w))
    res.update(dh=dh.to(dtype), dweight=(c["scale"] * (dz.t() @ x)).to(dtype))
    if c["bias"]:
        res["dbias"] = dz.sum(0)
    return res


# ---------------------------------------------------------------------------
# the definitions in 64 bits
def exact(case, seed):
    if case["op"] in ("loss", "loss_train") and work(case)["flops"] > 1.2e13:
        return None
    st = prepare(case, seed)
    if case["op"] in ("embed", "embed_train"):
        return _exact_embed(case, st)
    if case["op"] in ("step", "step_train"):
        return _exact_step(case, st)
    return _exact_loss(case, st)


def _exact_embed(case, st):
    ids = st["ids"].long()
    rows = torch.cat([st["table"].double() * st["scale"], torch.zeros(1, case["width"], dtype=torch.float64, device=DEV)])
    slot = torch.where((ids < 0) | (ids >= case["vocab"]), case["vocab"], ids)    # the last row is nobody's
    res = {"out": rows[slot]}
    if case["op"] == "embed_train":
        order = torch.argsort(slot, stable=True)
        count = torch.bincount(slot, minlength=case["vocab"] + 1)
        # sums over each word's stretch of the sorted rows, a width at a time
        step = max(1, 200_000_000 // max(1, case["tokens"]))
        parts = []
        for c in range(0, case["width"], step):
            d = st["dout"][:, c:c + step].double()[order] * st["scale"]
            parts.append(torch.segment_reduce(d, "sum", lengths=count, axis=0, initial=0.0)[:-1])
        res["dtable"] = torch.cat(parts, 1)
    return res


def _exact_step(case, st):
    def leaf(t):
        return None if t is None else t.detach().double().requires_grad_(case["op"] == "step_train")

    h, y, w2, b2, w1, b1, gate = (leaf(st[k]) for k in ("h", "y", "weight", "bias", "post_weight", "post_bias", "gate"))

    def norm(x, w, b):
        mu = 0.0 if case["rms"] else torch.mean(x, dim=-1, keepdim=True)
        var = torch.mean((x - mu) ** 2, dim=-1, keepdim=True)
        out = (x - mu) / torch.sqrt(var + EPS) * w
        return out if b is None else out + b

    u = norm(y, w1, b1) if case["post"] else y
    stream = h * case["alpha"] + (u if gate is None else u * gate)
    x = norm(stream, w2, b2) if case["pre"] else None
    res = {"stream": stream.detach()}
    if x is not None:
        res["x"] = x.detach()
    if case["op"] == "step_train":
        total = (stream * st["dstream"].double()).sum()
        if x is not None:
            total = total + (x * st["dx"].double()).sum()
        names = [("dh", h), ("dy", y), ("dweight", w2), ("dbias", b2), ("dpost_weight", w1), ("dpost_bias", b1), ("dgate", gate)]
        names = [(k, t) for k, t in names if t is not None]
        res.update(zip((k for k, _ in names), torch.autograd.grad(total, [t for _, t in names])))
    return res


def _exact_loss(case, st):
    n, v, d = case["rows"], case["classes"], case["width"]
    f64 = dict(dtype=torch.float64, device=DEV)
    rows = [r for r, t in enumerate(st["targets"].tolist()) if 0 <= t < v]
    rows = torch.tensor(rows, dtype=torch.int64, device=DEV)
    w = st["weight"].double()
    b = st["bias"].double() if case["bias"] else torch.zeros(v, **f64)
    loss, lse, dh = torch.zeros(n, **f64), torch.zeros(n, **f64), torch.zeros(n, d, **f64)
    dw, db = torch.zeros(v, d, **f64), torch.zeros(v, **f64)
    for r in rows.split(max(1, (1 << 28) // v)):
        x, t = st["h"][r].double(), st["targets"][r].long()
        z = torch.addmm(b, x, w.mT, alpha=case["scale"])
        lse[r] = torch.logsumexp(z, 1)
        own_z = z[torch.arange(len(r), device=DEV), t]
        loss[r] = lse[r] - own_z
        if case["op"] == "loss_train":
            p = torch.exp(z - lse[r][:, None])
            p[torch.arange(len(r), device=DEV), t] -= 1
            p *= st["dloss"][r].double()[:, None]
            dh[r] = torch.mm(p, w) * case["scale"]
            dw.addmm_(p.mT, x, alpha=case["scale"])
            db += p.sum(0)
    res = {"loss": loss, "lse": lse}
    if case["op"] == "loss_train":
        res.update(dh=dh, dweight=dw)
        if case["bias"]:
            res["dbias"] = db
    return res
