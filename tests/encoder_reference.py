"""The encoder operators from their definitions, in 64 bits, one document and
one head at a time, with elementwise bounds on what the kernels may be off by.

Bounds.  u is the unit roundoff of a type (2^-8 for bf16, 2^-11 for fp16,
2^-24 for fp32).  The attention kernels round a probability once to 16 bits
before the product with v (or dout), ds once before the products with q and
k, and every result once; everything else is fp32.  So
  |out error|  <= u (sum p |v| + |out|)                       + fp32 terms
  |dv error|   <= u (sum p |dout| + |dv|)                     + fp32 terms
  |delta error| <= e = sum |dout| |out error|
  |dq error|   <= scale sum (u |ds| + p e) |k| + u |dq|       + fp32 terms
  |dk error|   <= scale sum (u |ds| + p e) |q| + u |dk|       + fp32 terms
The fp32 terms: a score is a sum of head_dim products, off by at most
head_dim 2^-24 sum |q||k| scale in any order; with the exponential's own error
p is off by the relative amount r = 2 head_dim 2^-24 max(sum |q||k|) scale +
2^-20, and every sum above by r of its sum of magnitudes.  The table's
gradient has no rounding to 16 bits and an exact delta: its bound is
2 r sum p (|dp| + |delta|) over the pairs of the bucket.
"""
import math

import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 1e-37, torch.float16: 2.0 ** -24, torch.float32: 1e-37}   # about a subnormal step


def offsets_of(lengths, device):
    return torch.tensor([0] + list(lengths)).cumsum(0).to(torch.int32).to(device)


def attention(q, k, v, qlen, klen, table=None, buckets=None, causal=False, scale=None, dout=None):
    """q [tokens][heads][dim] etc. of any type.  Returns a dict of 64-bit
    results (out, lse; with dout also dq, dk, dv, dtable) and one of bounds."""
    dt = q.dtype
    u = U[dt]
    q, k, v = q.double(), k.double(), v.double()
    heads, share, d = q.shape[1], q.shape[1] // k.shape[1], q.shape[2]
    scale = d ** -0.5 if scale is None else scale
    dev = q.device
    res = {"out": torch.zeros_like(q), "lse": torch.full((heads, q.shape[0]), -math.inf, dtype=q.dtype, device=dev)}
    err = {"out": torch.zeros_like(q), "lse": torch.zeros_like(res["lse"])}
    if dout is not None:
        dout = dout.double()
        for name, t in (("dq", q), ("dk", k), ("dv", v)) + ((("dtable", table.double()),) if table is not None else ()):
            res[name], err[name] = torch.zeros_like(t), torch.zeros_like(t)
    q0 = k0 = 0
    for a, b in zip(qlen, klen):
        qs, ks = slice(q0, q0 + a), slice(k0, k0 + b)
        q0, k0 = q0 + a, k0 + b
        if not a or not b:
            continue
        dist = torch.arange(b, device=dev)[None] - torch.arange(a, device=dev)[:, None] - (b - a)
        for h in range(heads):
            qq, kk, vv = q[qs, h], k[ks, h // share], v[ks, h // share]
            s = scale * qq @ kk.T
            mag = abs(scale) * qq.abs() @ kk.abs().T
            if table is not None:
                reach = buckets.shape[0] // 2
                at = buckets.long()[dist.clamp(-reach, reach) + reach]
                s = s + table.double()[at, h]
            if causal:
                s = s.masked_fill(dist > 0, -math.inf)
            seen = s > -math.inf
            top = s.amax(1, keepdim=True)
            top = torch.where(top > -math.inf, top, 0.0)
            e = torch.where(seen, torch.exp(s - top), 0.0)
            z = e.sum(1, keepdim=True)
            p = e / torch.where(z > 0, z, 1.0)
            r = 2 * d * 2.0 ** -24 * (mag * seen).amax() + 2.0 ** -20
            out = p @ vv
            res["out"][qs, h] = out
            res["lse"][h, qs] = (top + torch.log(z))[:, 0]
            big = torch.where(seen, s.abs(), 0.0).amax()
            err["lse"][h, qs] = r + 2.0 ** -22 * min(float(big), 1e30)
            pv = p @ vv.abs()
            err_out = (u + 2 * r) * pv + u * out.abs() + TINY[dt]
            err["out"][qs, h] = err_out
            if dout is None:
                continue
            do = dout[qs, h]
            dp = do @ vv.T
            delta = (do * out).sum(1, keepdim=True)
            ds = p * (dp - delta)
            e_delta = (do.abs() * err_out).sum(1, keepdim=True)
            eds = u * ds.abs() + p * e_delta + 2 * r * p * (do.abs() @ vv.abs().T + delta.abs())
            res["dq"][qs, h] = scale * ds @ kk
            err["dq"][qs, h] = abs(scale) * (eds @ kk.abs() + 2 * r * ds.abs() @ kk.abs())
            res["dk"][ks, h // share] += scale * ds.T @ qq
            err["dk"][ks, h // share] += abs(scale) * (eds.T @ qq.abs() + 2 * r * ds.abs().T @ qq.abs())
            res["dv"][ks, h // share] += p.T @ do
            err["dv"][ks, h // share] += (u + 2 * r) * p.T @ do.abs()
            if table is not None:
                n = table.shape[0]
                res["dtable"][:, h] += torch.bincount(at.flatten(), ds.flatten(), n)
                err["dtable"][:, h] += 2 * r * torch.bincount(at.flatten(), (p * (dp.abs() + delta.abs())).flatten(), n)
    for name in ("dq", "dk", "dv"):
        if name in res:
            err[name] += u * res[name].abs() + TINY[dt]
    return res, err


def layer_norm(x, w, b, eps, dy=None):
    """64-bit results and bounds: with c = 2^-24 (the sums are trees of fp32
    additions over values held once), the mean is off by at most
    c' max|x|, c' = 2^-21, a centred value by that and its own rounding, and
    r relatively by as much; results round once to their type."""
    c = 2.0 ** -21
    dt = x.dtype
    wt = w.dtype
    x, w = x.double(), w.double()
    mu = x.mean(1, keepdim=True)
    r = 1 / ((x - mu).square().mean(1, keepdim=True) + eps).sqrt()
    xh = (x - mu) * r
    y = xh * w + (0 if b is None else b.double())
    exh = c * x.abs().amax(1, keepdim=True) * r + c * xh.abs()         # error of xh
    exh = exh * (1 + xh.abs())                                          # through the variance as well
    res = {"y": y, "mean": mu[:, 0], "rstd": r[:, 0]}
    err = {"y": exh * w.abs() + (U[dt] + c) * y.abs() + c * w.abs() + TINY[dt]}
    if dy is not None:
        dy = dy.double()
        g = dy * w
        n = x.shape[1]
        m1, m2 = g.mean(1, keepdim=True), (g * xh).mean(1, keepdim=True)
        res["dx"] = r * (g - m1 - xh * m2)
        ga, big = g.abs().mean(1, keepdim=True), exh.amax(1, keepdim=True)
        err["dx"] = r * (big * (g.abs() + ga) * 2 + c * (g.abs() + ga + xh.abs() * (g * xh).abs().mean(1, keepdim=True))
                         + xh.abs() * ga * big + exh * m2.abs()) + U[dt] * res["dx"].abs() + TINY[dt]
        res["dw"], res["db"] = (dy * xh).sum(0), dy.sum(0)
        err["dw"] = (dy.abs() * (exh + c * xh.abs())).sum(0) + U[wt] * res["dw"].abs() + TINY[wt]
        err["db"] = c * dy.abs().sum(0) + U[wt] * res["db"].abs() + TINY[wt]
        del n
    return res, err


def unit_pool(h, lengths, drows=None):
    """64-bit unit rows; fp32 sums over a document's tokens are off by at most
    2^-24 log-depth of the magnitudes: c = 2^-20 of the mean of |h|."""
    c = 2.0 ** -20
    dt = h.dtype
    h = h.double()
    rows, norms, erow, dh, edh = [], [], [], [], []
    start = 0
    for i, n in enumerate(lengths):
        x = h[start:start + n]
        start += n
        m = x.sum(0) / max(n, 1)
        em = c * x.abs().sum(0) / max(n, 1)
        size = m.norm()
        u = m / size if size > 0 else torch.zeros_like(m)
        eu = (em + u.abs() * em.norm()) / size + c * u.abs() if size > 0 else torch.zeros_like(m)
        rows.append(u)
        norms.append(size)
        erow.append(eu + 1e-37)
        if drows is not None and n:
            g = drows[i].double()
            d = (g - (g @ u) * u) / size / n if size > 0 else torch.zeros_like(m)
            ed = (g.norm() * (eu + u.abs() * eu.norm()) + (em.norm() / size + 8 * c) * (g.abs() + g.norm() * u.abs())) \
                / size / n if size > 0 else torch.zeros_like(m)
            dh.append(d.expand(n, -1))
            edh.append((ed + U[dt] * d.abs() + TINY[dt]).expand(n, -1))
    res = {"rows": torch.stack(rows), "norms": torch.stack(norms)}
    err = {"rows": torch.stack(erow)}
    if drows is not None:
        res["dh"], err["dh"] = torch.cat(dh), torch.cat(edh)
    return res, err


def assert_within(got, ref, bound, name):
    """Elementwise |got - ref| <= bound, infinities equal, no NaN."""
    got = got.double()
    assert got.shape == ref.shape, (name, got.shape, ref.shape)
    assert not got.isnan().any(), f"{name}: NaN"
    inf = ref.isinf()
    assert torch.equal(got[inf], ref[inf]) and not got[~inf].isinf().any(), f"{name}: infinities"
    over = ((got - ref).abs() - bound)[~inf]
    if over.numel() and over.max() > 0:
        at = torch.where((~inf) & ((got - ref).abs() > bound))
        i = tuple(x[0] for x in at)
        raise AssertionError(f"{name}: {at[0].numel()} of {got.numel()} outside their bounds, first at "
                             f"{[int(x) for x in i]}: {float(got[i])} against {float(ref[i])} +- {float(bound[i])}")
