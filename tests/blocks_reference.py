"""The operators around an encoder's blocks from their definitions, in 64 bits,
with elementwise bounds on what the kernels may be off by.

u is the unit roundoff of a type (encoder_reference.U).

Embedding: a product and one rounding.  Its gradient: fp32 additions, up to 64
one after the other, then up to a sixteenth of the id's pieces of 64, then 17:
that many times 2^-24 of the sum of magnitudes.

Residual norm: c = 2^-21 as for layer_norm; every error is carried on to first
order: of the normed y, the stream (which is not rounded between), its
statistics, and the gradients; the sums over rows add up to a 152th of the
rows one after the other and then at most 64 groups.

Cross entropy: a score is a sum of `width` products, off by at most 2 width
2^-24 sum |h||w| scale in any order (the tensor cores may cut off instead of
rounding), and a few roundings of its own and of the row's largest score; r is the
largest of these in a row, with 2^-20 for the exponential.  Then
  |lse error| <= r + 2^-22 |lse|,   |loss error| <= 3 r (1 - exp(-loss)) + 2^-20 loss
(the loss is log1p of a sum whose terms are off by 3 r at most, relatively),
  |q error| <= 3 r p, at the target the loss' error times exp(-loss),
and q is rounded once to 16 bits before the products, h times its row's dloss
over the largest once more where the rows' dloss differ.  A product's sum of m
terms is off by 2 m 2^-24 of the sum of magnitudes.
"""
import math

import torch

from encoder_reference import TINY, U, assert_within  # noqa: F401


def embed(ids, table, scale, dtype):
    ids = ids.long()
    real = (ids >= 0) & (ids < table.shape[0])
    res = torch.where(real[..., None], table.double()[torch.where(real, ids, 0)] * scale, 0.0)
    return res, (U[dtype] + 2.0 ** -24) * res.abs() + TINY[dtype]


def embed_backward(dout, ids, vocab, scale, dtype, old=None):
    ids = ids.flatten().long()
    d = dout.reshape(-1, dout.shape[-1]).double()
    real = (ids >= 0) & (ids < vocab)
    d, ids = d[real], ids[real]
    zero = torch.zeros(vocab, d.shape[1], dtype=torch.float64, device=d.device)
    res, mag = zero.index_add(0, ids, d * scale), zero.index_add(0, ids, d.abs() * abs(scale))
    count = torch.bincount(ids, minlength=vocab).double()[:, None]
    depth = count.clamp(max=64) + count / 1024 + 20
    err = depth * 2.0 ** -24 * mag
    if old is not None:
        res, touched = res + old.double(), count > 0
        err = torch.where(touched, err + 2.0 ** -23 * old.double().abs(), 0.0)
        return res, torch.where(touched, err + U[dtype] * res.abs() + TINY[dtype], 0.0)
    return res, err + U[dtype] * res.abs() + TINY[dtype] * (count > 0)


def _norm(v, ev, w, b, eps, rms):
    """Output, normed v, its factor; errors of the output, the normed v, and the factor (relative)."""
    c = 2.0 ** -21
    mu = torch.zeros_like(v[:, :1]) if rms else v.mean(1, keepdim=True)
    r = 1 / ((v - mu).square().mean(1, keepdim=True) + eps).sqrt()
    vh = (v - mu) * r
    e = ev + (0 if rms else ev.mean(1, keepdim=True)) + c * v.abs().amax(1, keepdim=True)
    er = r * (vh.abs() * e).mean(1, keepdim=True) + c
    evh = r * e + 2 * vh.abs() * er
    out = vh * w + (0 if b is None else b)
    return out, vh, r, evh * w.abs() + c * (out.abs() + (vh * w).abs()), evh, er


def residual_norm(h, y, weight=None, bias=None, post_weight=None, post_bias=None, gate=None, alpha=1.0, eps=1e-5,
                  rms=False, dstream=None, dx=None):
    """64-bit results and bounds by name; the gradients where dstream or dx is given."""
    c, dt = 2.0 ** -21, h.dtype
    wt = (weight if weight is not None else post_weight).dtype

    def d(t):
        return None if t is None else t.double()

    h, y, w2, b2, w1, b1, g = (d(t) for t in (h, y, weight, bias, post_weight, post_bias, gate))
    u, eu, yh, eyh, r1, er1 = y, torch.zeros_like(y), y, torch.zeros_like(y), 1.0, 0.0
    if w1 is not None:
        u, yh, r1, eu, eyh, er1 = _norm(y, torch.zeros_like(y), w1, b1, eps, rms)
    gate64 = torch.ones_like(h[0]) if g is None else g
    s = alpha * h + gate64 * u
    es = gate64.abs() * eu + c * ((alpha * h).abs() + (gate64 * u).abs())
    res, err = {"stream": s}, {"stream": es}
    if w2 is not None:
        x, sh, r2, ex, esh, er2 = _norm(s, es, w2, b2, eps, rms)
        res["x"], err["x"] = x, ex
    if dstream is not None or dx is not None:
        G = torch.zeros_like(h) if dstream is None else dstream.double()
        eG = c * G.abs()
        depth = (h.shape[0] / 152 + 65) * 2.0 ** -24

        def back(d, ed, vh, evh, r, er):
            m1 = 0.0 if rms else d.mean(1, keepdim=True)
            a1 = d.abs().mean(1, keepdim=True)
            m2 = (d * vh).mean(1, keepdim=True)
            out = r * (d - m1 - vh * m2)
            e = r * (ed + ed.mean(1, keepdim=True) + c * (d.abs() + a1) + evh * m2.abs()
                     + vh.abs() * ((ed * vh.abs() + d.abs() * evh).mean(1, keepdim=True)
                                   + 2 * c * (d * vh).abs().mean(1, keepdim=True)))
            return out, e + er * (r * (d.abs() + a1 + (vh * m2).abs()))

        if w2 is not None:
            dx = dx.double()
            back2, eback2 = back(dx * w2, c * (dx * w2).abs(), sh, esh, r2, er2)
            G, eG = G + back2, eG + eback2 + c * (G.abs() + back2.abs())
            res["dweight"], err["dweight"] = (dx * sh).sum(0), (dx.abs() * (esh + (depth + c) * sh.abs())).sum(0)
            if b2 is not None:
                res["dbias"], err["dbias"] = dx.sum(0), depth * dx.abs().sum(0)
        res["dh"], err["dh"] = alpha * G, abs(alpha) * eG + c * (alpha * G).abs()
        du, edu = gate64 * G, gate64.abs() * eG + c * (gate64 * G).abs()
        eGu = eG * u.abs() + G.abs() * eu + 2 * c * (G * u).abs()
        if w1 is not None:
            res["dy"], err["dy"] = back(du * w1, edu * w1.abs() + c * (du * w1).abs(), yh, eyh, r1, er1)
            res["dpost_weight"] = (du * yh).sum(0)
            err["dpost_weight"] = (edu * yh.abs() + du.abs() * eyh + (depth + 2 * c) * (du * yh).abs()).sum(0)
            if b1 is not None:
                res["dpost_bias"], err["dpost_bias"] = du.sum(0), (edu + (depth + 2 * c) * du.abs()).sum(0)
        else:
            res["dy"], err["dy"] = du, edu
        if g is not None and g.dim() == 1:
            # added up as w sum(G yh) + b sum(G)
            parts = (G * yh).abs() * (1 if w1 is None else w1.abs()) + (0 if b1 is None else (G * b1).abs())
            res["dgate"], err["dgate"] = (G * u).sum(0), (eGu + eG * (0 if b1 is None else b1.abs())
                                                          + eG * (yh.abs() * (1 if w1 is None else w1.abs()))
                                                          + (depth + 2 * c) * parts).sum(0)
        elif g is not None:
            res["dgate"], err["dgate"] = G * u, eGu
    columns = ("dweight", "dbias", "dpost_weight", "dpost_bias") + (("dgate",) if g is not None and g.dim() == 1 else ())
    for name in res:
        t = wt if name in columns else dt
        err[name] = err[name] + U[t] * res[name].abs() + TINY[t]
    return res, err


def cross_entropy(h, weight, targets, bias=None, scale=1.0, dloss=None, dweight_dtype=None, old=None):
    """64-bit results and bounds by name."""
    dt, u = h.dtype, U[h.dtype]
    n, width = h.shape
    classes = weight.shape[0]
    t = targets.long()
    live = (t >= 0) & (t < classes)
    x, w, t = h[live].double(), weight.double(), t[live]
    b = torch.zeros(classes, dtype=torch.float64, device=h.device) if bias is None else bias.double()
    hidden = b < -1e30
    z = scale * x @ w.T + b
    big = torch.where(hidden, 0.0, z.abs() + b.abs()).amax(1)
    r = (2 * width * 2.0 ** -24 * abs(scale) * (x.abs() @ w.abs().T).amax(1) + 2.0 ** -21 * big + 2.0 ** -20)[:, None]
    top = z.amax(1, keepdim=True)
    seen = torch.isfinite(top)
    e = torch.where(seen, torch.exp(z - torch.where(seen, top, 0.0)), 0.0)
    total = e.sum(1, keepdim=True)
    lse = top + torch.log(total)
    p = torch.where(seen, e / torch.where(seen, total, 1.0), 0.0)
    hit = z.gather(1, t[:, None])
    others = torch.where(seen, e.scatter(1, t[:, None], 0.0).sum(1, keepdim=True), 0.0)
    loss = torch.where(torch.isneginf(hit), math.inf,
                       torch.log1p(others / torch.where(seen, torch.exp(hit - top), 1.0)))
    loss = torch.where(torch.isfinite(loss) | torch.isneginf(hit), loss, (lse - hit))
    away = -torch.expm1(-loss)                                         # 1 - the target's probability
    eloss = torch.where(torch.isfinite(loss), 3 * r * away + 2.0 ** -20 * torch.where(torch.isfinite(loss), loss, 0.0) + 1e-37, 0.0)
    at = live.nonzero()[:, 0]
    zero = torch.zeros(n, dtype=torch.float64, device=h.device)
    res = {"loss": zero.index_copy(0, at, loss[:, 0]), "lse": zero.index_copy(0, at, lse[:, 0])}
    err = {"loss": zero.index_copy(0, at, eloss[:, 0]),
           "lse": zero.index_copy(0, at, (r + 2.0 ** -22 * torch.where(torch.isfinite(lse), lse.abs(), 0.0))[:, 0])}
    if dloss is None:
        return res, err
    g = dloss[live].double()[:, None]
    q = p.scatter(1, t[:, None], -away)
    eq = (3 * r * p).scatter(1, t[:, None], (1 - away) * eloss) + 2.0 ** -22 * q.abs() + (2.0 ** -39 if dt == torch.float16 else 0.0)
    eq16 = eq + u * q.abs()
    dh = torch.zeros(n, width, dtype=torch.float64, device=h.device)
    res["dh"] = dh.index_copy(0, at, scale * (g * q) @ w)
    err["dh"] = dh.index_copy(0, at, abs(scale) * g.abs() * ((eq16 + 2 * classes * 2.0 ** -24 * q.abs()) @ w.abs()))
    err["dh"] += (u + 2.0 ** -22) * res["dh"].abs() + TINY[dt]
    m = max(1, len(at))
    res["dweight"] = scale * (g * q).T @ x
    differ = len(at) > 0 and bool((g != g[0]).any())
    err["dweight"] = abs(scale) * (g.abs() * (eq16 + 2 * m * 2.0 ** -24 * q.abs() + (u * q.abs() if differ else 0.0))).T @ x.abs()
    if differ and dt == torch.float16:
        err["dweight"] += abs(scale) * float(g.abs().max()) * TINY[dt] * q.abs().sum(0)[:, None]
    wt = weight.dtype if dweight_dtype is None else dweight_dtype
    if old is not None:
        res["dweight"] = res["dweight"] + old.double()
        err["dweight"] += 2.0 ** -24 * old.double().abs()
    err["dweight"] += (U[wt] + 2.0 ** -22) * res["dweight"].abs() + TINY[wt]
    if bias is not None:
        res["dbias"] = (g * q).sum(0)
        err["dbias"] = (g.abs() * (eq + (m + 4) * 2.0 ** -24 * q.abs())).sum(0) + 1e-37
    return res, err
