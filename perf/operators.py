"""The measured work of the encoder operators: what turns packed documents
into the unit rows that the deduplication search takes, and its training.

A program keeps its documents packed one after the other (no padding), with
the offsets of their first rows, runs layer norm and attention with a learned
relative position bias over them, and pools every document into one unit row.  Training
runs the backward passes too.  Each case below is one such call (a training
case: the forward call and its backward call).  Lengths are part of the case;
values come from the seed.
"""
import math
import random

import torch

own = False

DEV = "cuda"
EPS = 1e-5
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def listed():
    return [
        # the rows of one short text on its way to the search: pure latency
        dict(name="norm_text", op="norm", rows=23, width=768, dtype="bf16", weights="bf16", bias=True),
        # a corpus batch, inference
        dict(name="norm_corpus", op="norm", rows=200_003, width=1024, dtype="bf16", weights="fp32", bias=True),
        # the same in training: output, input gradient, weight and bias gradient
        dict(name="norm_train", op="norm_train", rows=100_003, width=768, dtype="bf16", weights="bf16", bias=True),
        # an odd width in 32 bits, no bias
        dict(name="norm_odd", op="norm_train", rows=20_011, width=1001, dtype="fp32", weights="fp32", bias=False),
        # one short text through attention: pure latency
        dict(name="attend_text", op="attend", nseq=1, lo=23, hi=23, new=0, heads=12, kv_heads=12, dim=64,
             buckets=32, reach=128, causal=False, dtype="fp16"),
        # a batch of documents of 0 to 512 tokens, looking both ways
        dict(name="attend_docs", op="attend", nseq=512, lo=0, hi=512, new=0, heads=12, kv_heads=12, dim=64,
             buckets=32, reach=128, causal=False, dtype="bf16"),
        # long documents under a causal encoder with shared key heads, no bias
        dict(name="attend_long", op="attend", nseq=4, lo=6001, hi=8192, new=0, heads=16, kv_heads=4, dim=128,
             buckets=0, reach=0, causal=True, dtype="bf16"),
        # one more token for each of many growing documents
        dict(name="attend_token", op="attend", nseq=24, lo=1, hi=32_768, new=1, heads=16, kv_heads=4, dim=128,
             buckets=32, reach=128, causal=True, dtype="bf16"),
        # a training batch of documents
        dict(name="train_docs", op="attend_train", nseq=384, lo=0, hi=512, new=0, heads=12, kv_heads=12, dim=64,
             buckets=32, reach=128, causal=False, dtype="bf16"),
        # training on long documents
        dict(name="train_long", op="attend_train", nseq=3, lo=3001, hi=8192, new=0, heads=16, kv_heads=4, dim=128,
             buckets=0, reach=0, causal=True, dtype="bf16"),
        # the unit rows of a batch of documents
        dict(name="pool_docs", op="pool", nseq=2048, lo=0, hi=512, width=768, dtype="bf16"),
        # and in training: rows and the gradient of every token
        dict(name="pool_train", op="pool_train", nseq=500, lo=1, hi=4096, width=256, dtype="fp32"),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm_train", "attend", "attend", "attend", "attend_train", "attend_train", "pool",
                     "pool_train"])
    if op in ("norm", "norm_train"):
        width = rng.choice([64, 96, 256, 384, 512, 768, 1024, 2048, _spread(rng, 1, 4096)])
        dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
        top = min(200_000, 75_000_000 // width // (2 if dtype == "fp32" else 1))
        return dict(op=op, rows=_spread(rng, 1, top), width=width, dtype=dtype,
                    weights=rng.choice([dtype, "fp32"]), bias=rng.random() < 0.7)
    if op in ("pool", "pool_train"):
        width = rng.choice([96, 256, 512, 768, 1024, _spread(rng, 4, 1024)])
        hi = _spread(rng, 4, 8192)
        nseq = max(1, min(_spread(rng, 1, 4096), 150_000_000 // (hi * width)))
        return dict(op=op, nseq=nseq, lo=rng.choice([0, 1, hi // 2]), hi=hi, width=width,
                    dtype=rng.choice(["bf16", "fp16", "fp32"]))
    dim = rng.choice([32, 64, 64, 80, 96, 128, 128])
    kv_heads = rng.choice([1, 2, 4, 6, 12])
    heads = kv_heads * rng.choice([1, 1, 2, 3, 4, 8])
    new = rng.choice([1, 1, 4]) if op == "attend" and rng.random() < 0.35 else 0
    hi = _spread(rng, 16, 32_768 if new else 8192)
    lo = rng.choice([0, 1, hi // 2, hi])
    # no drawn batch costs more than the largest listed one
    pairs = heads * hi * (new or hi)
    most = min(3e9, 1.2e12 / (dim * (14 if op == "attend_train" else 4)))
    heads = heads if pairs < most else kv_heads
    hi = hi if pairs < most else min(hi, 4096)
    lo = min(lo, hi)
    nseq = int(max(1, min(_spread(rng, 1, 1024), most // (heads * hi * (new or hi)),
                          110_000_000 // (hi * (kv_heads + (0 if new else heads)) * dim))))
    buckets = rng.choice([0, 16, 32, 32, 64])
    return dict(op=op, nseq=nseq, lo=lo, hi=hi, new=new, heads=heads, kv_heads=kv_heads, dim=dim, buckets=buckets,
                reach=rng.choice([64, 128, 128, 256]) if buckets else 0, causal=bool(new) or rng.random() < 0.5,
                dtype=rng.choice(["bf16", "bf16", "fp16"]))


def _lengths(case):
    """The documents' lengths: part of the case, spread between its bounds,
    the longest and the shortest present."""
    lo, hi, nseq = case["lo"], case["hi"], case["nseq"]
    rng = random.Random(f"{nseq}/{lo}/{hi}")
    out = [int(round(lo + (hi - lo) * rng.random() ** 1.5)) for _ in range(nseq)]
    out[0] = hi
    if nseq > 1:
        out[nseq // 2] = lo
    return out


def _query_lengths(case):
    """New tokens against everything kept of their document, or each document against itself."""
    return [case["new"]] * case["nseq"] if case["new"] else _lengths(case)


def _pairs(case):
    """Pairs of a query and a key it sees: a causal query at place i of its
    `a` sees all but the last a - 1 - i keys of its document."""
    return sum(max(0, b - (a - 1 - i)) for a, b in zip(_query_lengths(case), _lengths(case)) for i in range(a)) \
        if case["causal"] else sum(a * b for a, b in zip(_query_lengths(case), _lengths(case)))


def work(case):
    size = 4 if case["dtype"] == "fp32" else 2
    if case["op"] in ("norm", "norm_train"):
        n, w = case["rows"], case["width"]
        wsize = 4 if case["weights"] == "fp32" else 2
        nw = 2 if case["bias"] else 1
        if case["op"] == "norm":
            return {"bytes": 2 * n * w * size + nw * w * wsize, "flops": 8 * n * w}
        return {"bytes": 4 * n * w * size + 2 * nw * w * wsize, "flops": 20 * n * w}
    if case["op"] in ("pool", "pool_train"):
        tokens, w = sum(_lengths(case)), case["width"]
        if case["op"] == "pool":
            return {"bytes": tokens * w * size + case["nseq"] * w * 4, "flops": tokens * w + 3 * case["nseq"] * w}
        return {"bytes": 2 * tokens * w * size + 2 * case["nseq"] * w * 4, "flops": tokens * w + 8 * case["nseq"] * w}
    q = sum(_query_lengths(case)) * case["heads"] * case["dim"]
    k = sum(_lengths(case)) * case["kv_heads"] * case["dim"]
    table = case["buckets"] * case["heads"] * 4
    pairs = _pairs(case) * case["heads"]
    if case["op"] == "attend":
        return {"bytes": (2 * q + 2 * k) * size + table, "flops": 4 * case["dim"] * pairs}
    return {"bytes": (4 * q + 4 * k) * size + 2 * table, "flops": 14 * case["dim"] * pairs}


# ---------------------------------------------------------------------------
# what a program has in hand
def _bucket(distance, case):
    """The bucket of a signed distance key - query.  Near ones have their own;
    farther ones share buckets whose bounds grow geometrically up to `reach`.
    A causal encoder keeps all buckets for the keys behind."""
    half = case["buckets"] if case["causal"] else case["buckets"] // 2
    base = half if not case["causal"] and distance > 0 else 0
    n = max(0, -distance) if case["causal"] else abs(distance)
    near = half // 2
    far = half - near
    # t steps out where (n / near)^far >= (reach / near)^t, in whole numbers
    return base + (n if n < near else near + sum(n ** far * near ** t >= case["reach"] ** t * near ** far
                                                 for t in range(1, far)))


def prepare(case, seed):
    g = torch.Generator(DEV).manual_seed(seed)
    dtype = DTYPES[case["dtype"]]

    def randn(*shape):
        return torch.randn(*shape, generator=g, device=DEV)

    st = {"case": case}
    if case["op"] in ("norm", "norm_train"):
        n, w = case["rows"], case["width"]
        wd = DTYPES[case["weights"]]
        # hidden states: channels of unequal spread around their own means
        spread = torch.exp(0.5 * randn(w))
        st["x"] = (randn(n, w) * spread + 0.3 * randn(w)).to(dtype)
        st["weight"] = (1 + 0.1 * randn(w)).to(wd)
        st["bias"] = (0.1 * randn(w)).to(wd) if case["bias"] else None
        if case["op"] == "norm_train":
            st["dy"] = randn(n, w).to(dtype)
        return st
    if case["op"] in ("pool", "pool_train"):
        lengths = _lengths(case)
        st["h"] = (randn(sum(lengths), case["width"]) + randn(case["width"])).to(dtype)
        st["offsets"] = _offsets(lengths)
        if case["op"] == "pool_train":
            st["drows"] = randn(case["nseq"], case["width"])
        return st
    nq, nk = sum(_query_lengths(case)), sum(_lengths(case))
    d, h, hk = case["dim"], case["heads"], case["kv_heads"]
    st["q"] = (1.5 * randn(nq, h, d)).to(dtype)
    if case["new"]:
        st["k"], st["v"] = randn(nk, hk, d).to(dtype), randn(nk, hk, d).to(dtype)
    else:
        # one projection holds keys and values
        kv = randn(nk, 2, hk, d).to(dtype)
        st["k"], st["v"] = kv[:, 0], kv[:, 1]
    st["table"] = 0.7 * randn(case["buckets"], h) if case["buckets"] else None
    if case["op"] == "attend_train":
        st["dout"] = randn(nq, h, d).to(dtype)
    if case["new"]:
        st["q"] = st["q"].view(case["nseq"], case["new"], h, d)
    # where each document starts among the packed rows, and where the last ends
    st["offsets"] = _offsets(_lengths(case))
    r = case["reach"]
    st["map"] = torch.tensor([_bucket(t, case) for t in range(-r, r + 1)], dtype=torch.int32).to(DEV) if r else None
    return st


def _offsets(lengths):
    return torch.tensor([0] + lengths).cumsum(0).to(torch.int32).to(DEV)


# ---------------------------------------------------------------------------
# one pass
def run(st):
    op = st["case"]["op"]
    if op in ("norm", "norm_train"):
        return _own_norm(st) if own else _plain_norm(st)
    if op in ("pool", "pool_train"):
        return _own_pool(st) if own else _plain_pool(st)
    return _own_attend(st) if own else _plain_attend(st)


def _own_norm(st):
    import paper_2608_03199_gb300 as sieve
    y, mean, rstd = sieve.layer_norm(st["x"], st["weight"], st["bias"], eps=EPS)
    if st["case"]["op"] == "norm":
        return {"y": y}
    dx, dw, db = sieve.layer_norm_backward(st["dy"], st["x"], st["weight"], mean, rstd,
                                           need_dbias=st["case"]["bias"])
    return {"y": y, "dx": dx, "dweight": dw, "dbias": db} if st["case"]["bias"] else {"y": y, "dx": dx, "dweight": dw}


def _own_pool(st):
    import paper_2608_03199_gb300 as sieve
    rows, norms = sieve.unit_pool(st["h"], st["offsets"])
    if st["case"]["op"] == "pool":
        return {"rows": rows}
    return {"rows": rows, "dh": sieve.unit_pool_backward(st["drows"], rows, norms, st["offsets"], st["h"].shape[0],
                                                         dtype=st["h"].dtype)}


def _own_attend(st):
    import paper_2608_03199_gb300 as sieve
    c = st["case"]
    kw = dict(table=st["table"], buckets=st["map"], causal=c["causal"])
    out, lse = sieve.attention(st["q"], st["k"], st["v"], st["offsets"], **kw)
    if c["op"] == "attend":
        return {"out": out, "lse": lse}
    dq, dk, dv, dtable = sieve.attention_backward(st["dout"], st["q"], st["k"], st["v"], out, lse, st["offsets"], **kw)
    grads = {"out": out, "dq": dq, "dk": dk, "dv": dv}
    if c["buckets"]:
        grads["dtable"] = dtable
    return grads


def _plain_norm(st):
    x = st["x"].float()
    w = st["weight"].float()
    centred = x - x.mean(1, keepdim=True)
    rstd = 1 / torch.sqrt((centred * centred).mean(1, keepdim=True) + EPS)
    xh = centred * rstd
    y = xh * w
    if st["bias"] is not None:
        y = y + st["bias"].float()
    y = y.to(st["x"].dtype)
    if st["case"]["op"] == "norm":
        return {"y": y}
    dy = st["dy"].float()
    g = dy * w
    dx = rstd * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    out = {"y": y, "dx": dx.to(st["x"].dtype), "dweight": (dy * xh).sum(0).to(st["weight"].dtype)}
    if st["bias"] is not None:
        out["dbias"] = dy.sum(0).to(st["bias"].dtype)
    return out


def _plain_pool(st):
    h, n = st["h"].float(), st["offsets"].diff().long()
    owner = torch.repeat_interleave(torch.arange(len(n), device=DEV), n, output_size=h.shape[0])
    total = torch.zeros(len(n), h.shape[1], device=DEV).index_add_(0, owner, h)
    mean = total / n.clamp(min=1)[:, None]
    norm = mean.square().sum(1, keepdim=True).sqrt()
    inv = torch.where(norm > 0, 1 / norm, 0.0)
    rows = mean * inv
    if st["case"]["op"] == "pool":
        return {"rows": rows}
    g = st["drows"]
    dm = (g - (g * rows).sum(1, keepdim=True) * rows) * inv / n.clamp(min=1)[:, None]
    return {"rows": rows, "dh": dm[owner].to(st["h"].dtype)}


def _plain_attend(st):
    """Documents padded to the longest one: scores, a mask, exp and products."""
    c = st["case"]
    h, hk, d, n = c["heads"], c["kv_heads"], c["dim"], c["nseq"]
    dtype, scale = st["q"].dtype, 1 / math.sqrt(c["dim"])
    start, nk = st["offsets"][:-1].long()[:, None], st["offsets"].diff().long()[:, None]
    b = c["hi"]
    a = c["new"] or b
    row, col = torch.arange(a, device=DEV), torch.arange(b, device=DEV)
    real_k = col < nk                                                    # [n][b]
    ki = torch.where(real_k, start + col, 0)
    if c["new"]:
        real_q, qi = torch.ones(n, a, dtype=torch.bool, device=DEV), torch.arange(n * a, device=DEV).view(n, a)
        nq = torch.full_like(nk, a)
    else:
        real_q, qi, nq = real_k, ki, nk

    def padded(x, rows, real):                                           # [n][heads][rows][d]
        return (x[rows].float() * real[:, :, None, None]).transpose(1, 2)

    def groups(x):                                                       # heads of one group as rows of one product
        return x.reshape(n, hk, h // hk * x.shape[2], x.shape[3])

    q = padded(st["q"].reshape(-1, h, d), qi, real_q)
    k, v = padded(st["k"], ki, real_k), padded(st["v"], ki, real_k)
    dist = col - row[:, None] - (nk - nq)[:, :, None]                    # [n][a][b]
    seen = real_q[:, :, None] & real_k[:, None, :]
    if c["causal"]:
        seen = seen & (dist <= 0)
    s = (groups(q) @ k.transpose(2, 3)).view(n, h, a, b)
    s *= scale
    if c["buckets"]:
        near = dist[:1] if not c["new"] else dist                        # a document against itself: the same for all
        s += st["table"].t()[:, st["map"].long()[near.clamp(-c["reach"], c["reach"]) + c["reach"]]].transpose(0, 1)
    s.masked_fill_(~seen[:, None], -math.inf)
    top = s.amax(3, keepdim=True).clamp(min=-3e38)
    p = torch.exp_(s.sub_(top))
    z = p.sum(3, keepdim=True)
    p /= torch.where(z > 0, z, 1.0)
    o = (groups(p) @ v).view(n, h, a, d)
    total = (top + torch.log(z))[..., 0]
    out = o.transpose(1, 2)[real_q].to(dtype)
    if c["op"] == "attend":
        return {"out": out.view(st["q"].shape), "lse": total.transpose(1, 2)[real_q].t().contiguous()}
    do = padded(st["dout"], qi, real_q)
    dv = groups(p).transpose(2, 3) @ groups(do)
    ds = (groups(do) @ v.transpose(2, 3)).view(n, h, a, b)
    ds -= (do * o).sum(3, keepdim=True)
    ds *= p
    dq = (groups(ds) @ k).view(n, h, a, d) * scale
    dk = (groups(ds).transpose(2, 3) @ groups(q)) * scale
    grads = {"out": out, "dq": dq.transpose(1, 2)[real_q].to(dtype), "dk": dk.transpose(1, 2)[real_k].to(dtype),
             "dv": dv.transpose(1, 2)[real_k].to(dtype)}
    if c["buckets"]:
        # sums along the diagonals first, then over the distances of a bucket
        diagonal = (col - row[:, None] + a - 1).flatten()
        sums = torch.zeros(a + b - 1, h, device=DEV).index_add_(0, diagonal, ds.sum(0).flatten(1).t())
        at = st["map"].long()[torch.arange(1 - a, b, device=DEV).clamp(-c["reach"], c["reach"]) + c["reach"]]
        grads["dtable"] = torch.zeros(c["buckets"], h, device=DEV).index_add_(0, at, sums)
    return grads


# ---------------------------------------------------------------------------
# the definitions in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] in ("norm", "norm_train"):
        return _exact_norm(case, st)
    if case["op"] in ("pool", "pool_train"):
        return _exact_pool(case, st)
    cost = 2.0 * work(case)["flops"] * (2 if case["causal"] else 1)
    return _exact_attend(case, st) if cost < 1.5e13 else None


def _exact_norm(case, st):
    x, w = st["x"].double(), st["weight"].double()
    b = st["bias"].double() if case["bias"] else torch.zeros_like(w)
    var, mu = torch.var_mean(x, 1, correction=0, keepdim=True)
    sd = (var + EPS).sqrt()
    unit = (x - mu) / sd
    res = {"y": torch.addcmul(b, unit, w)}
    if case["op"] == "norm_train":
        dy = st["dy"].double()
        up = dy * w
        n = case["width"]
        along = (up * unit).sum(1, keepdim=True) / n
        res["dx"] = (up - up.sum(1, keepdim=True) / n - unit * along) / sd
        res["dweight"] = torch.einsum("rc,rc->c", dy, unit)
        if case["bias"]:
            res["dbias"] = dy.sum(0)
    return res


def _exact_pool(case, st):
    rows, grads = [], []
    start = 0
    for i, n in enumerate(_lengths(case)):
        h = st["h"][start:start + n].double()
        start += n
        m = h.sum(0) / max(n, 1)
        size = torch.linalg.vector_norm(m)
        u = torch.where(size > 0, m / size, torch.zeros_like(m))
        rows.append(u)
        if case["op"] == "pool_train" and n:
            g = st["drows"][i].double()
            dm = torch.where(size > 0, (g - torch.dot(g, u) * u) / size, torch.zeros_like(m))
            grads.append((dm / n).expand(n, -1))
    res = {"rows": torch.stack(rows)}
    if case["op"] == "pool_train":
        res["dh"] = torch.cat(grads) if grads else torch.zeros_like(st["h"], dtype=torch.float64)
    return res


def _exact_attend(case, st):
    h, d = case["heads"], case["dim"]
    share = h // case["kv_heads"]
    train = case["op"] == "attend_train"
    reach = case["reach"]
    queries = st["q"].view(-1, h, d)
    out = torch.zeros(queries.shape, dtype=torch.float64, device=DEV)
    lse = torch.full((h, queries.shape[0]), -math.inf, dtype=torch.float64, device=DEV)
    if train:
        dq, dk, dv = (torch.zeros(st[x].shape, dtype=torch.float64, device=DEV) for x in ("q", "k", "v"))
        dtable = torch.zeros(case["buckets"], h, dtype=torch.float64, device=DEV)
    bucket = torch.tensor([_bucket(t, case) for t in range(-reach, reach + 1)], device=DEV) if case["buckets"] else None
    q0 = k0 = 0
    for a, b in zip(_query_lengths(case), _lengths(case)):
        qs, ks = slice(q0, q0 + a), slice(k0, k0 + b)
        q0, k0 = q0 + a, k0 + b
        if not a or not b:
            continue
        dist = torch.arange(b, device=DEV)[None, :] - (torch.arange(a, device=DEV)[:, None] + b - a)
        step = max(1, (1 << 27) // (a * b))
        for i in range(0, h, step):
            hs = slice(i, min(i + step, h))
            kv = [j // share for j in range(hs.start, hs.stop)]
            q = queries[qs, hs].double().permute(1, 0, 2)
            k, v = (st[x][ks][:, kv].double().permute(1, 0, 2) for x in ("k", "v"))
            s = torch.baddbmm(torch.zeros((), dtype=torch.float64, device=DEV), q, k.mT, beta=0, alpha=d ** -0.5)
            if case["buckets"]:
                at = bucket[dist.clamp(-reach, reach) + reach]
                s += st["table"][:, hs].double().t()[:, at]
            if case["causal"]:
                s = torch.where(dist > 0, -math.inf, s)
            total = torch.logsumexp(s, 2)
            lse[hs, qs] = total
            # a query that sees no key answers with zeros
            p = torch.exp(s - torch.where(total.isneginf(), 0, total)[..., None])
            o = torch.bmm(p, v)
            out[qs, hs] = o.permute(1, 0, 2)
            if not train:
                continue
            do = st["dout"][qs, hs].double().permute(1, 0, 2)
            ds = p * (torch.bmm(do, v.mT) - torch.linalg.vecdot(do, o)[..., None])
            dq[qs, hs] = torch.bmm(ds, k).permute(1, 0, 2) * d ** -0.5
            gk, gv = torch.bmm(ds.mT, q) * d ** -0.5, torch.bmm(p.mT, do)
            for n, j in enumerate(kv):
                dk[ks, j] += gk[n]
                dv[ks, j] += gv[n]
                if case["buckets"]:
                    dtable[:, hs.start + n] += torch.bincount(at.flatten(), ds[n].flatten(), case["buckets"])
    if not train:
        return {"out": out.view(st["q"].shape), "lse": lse}
    res = {"out": out, "dq": dq, "dk": dk, "dv": dv}
    if case["buckets"]:
        res["dtable"] = dtable
    return res
