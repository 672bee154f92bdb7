"""The operators around an encoder's blocks on the GPU against their
definitions in 64 bits (blocks_reference)."""
import math

import pytest
import torch

import blocks_reference as ref
import paper_2608_03199_gb300 as sieve
from test_gpu_encoder import BF16, DEV, FP16, FP32, gen, randn

pytestmark = pytest.mark.gpu
I32, I64 = torch.int32, torch.int64


# ---------------------------------------------------------------- embedding
def zipf(g, n, vocab):
    """Ids as often as words in text."""
    u = torch.rand(n, generator=g, device=DEV).double()
    return torch.exp(u * math.log(vocab + 1)).long().sub_(1).clamp_(0, vocab - 1)


EMBED = [
    # tokens, vocab, width, table and gradient type, hidden type, id type
    (1, 1, 1, FP32, FP32, I64), (1, 7, 8, BF16, BF16, I32), (23, 50_000, 768, BF16, BF16, I64), (64, 5, 40, FP16, FP16, I32),
    (65, 5, 40, FP32, BF16, I64), (700, 511, 96, FP32, FP16, I32), (700, 512, 301, FP32, FP32, I64), (2049, 513, 257, BF16, FP32, I32),
    (5000, 3, 1000, FP16, BF16, I64), (9001, 100_003, 64, FP32, FP32, I64), (40_000, 262_144, 48, BF16, BF16, I32),
    (40_000, 3_000, 768, FP32, BF16, I64), (30_011, 1_000, 512, BF16, BF16, I32), (21_000, 5_000, 1_280, FP16, FP32, I64),
    (3, 20, 16_384, FP32, BF16, I32), (130, 9, 16_383, BF16, BF16, I64), (20_000, 1, 8, FP32, BF16, I64), (640_001, 300, 24, FP32, BF16, I32),
]


@pytest.mark.parametrize("tokens,vocab,width,ttype,dtype,itype", EMBED)
@pytest.mark.parametrize("scale,pad", [(1.0, 0.0), (-2.5, 0.3)])
def test_embed(tokens, vocab, width, ttype, dtype, itype, scale, pad):
    g = gen(tokens + width)
    ids = zipf(g, tokens, vocab)
    lost = torch.rand(tokens, generator=g, device=DEV) < pad
    outside = torch.tensor([-1, vocab, -2**31, 2**31 - 1], device=DEV)[torch.randint(4, (tokens,), generator=g, device=DEV)]
    ids = torch.where(lost, outside, ids).to(itype)
    table = randn(g, vocab, width).to(ttype)
    out = sieve.embed(ids, table, scale=scale, dtype=dtype)
    want, bound = ref.embed(ids, table, scale, dtype)
    assert out.dtype == dtype
    ref.assert_within(out, want, bound, "out")
    dout = randn(g, tokens, width).to(dtype)
    dtable = sieve.embed_backward(dout, ids, vocab, scale=scale, dtype=ttype)
    want, bound = ref.embed_backward(dout, ids, vocab, scale, ttype)
    assert dtable.dtype == ttype
    ref.assert_within(dtable, want, bound, "dtable")
    assert torch.equal(dtable, sieve.embed_backward(dout, ids, vocab, scale=scale, dtype=ttype))
    old = randn(g, vocab, width).to(ttype)
    total = old.clone()
    assert sieve.embed_backward(dout, ids, vocab, scale=scale, out=total, accumulate=True) is total
    want, bound = ref.embed_backward(dout, ids, vocab, scale, ttype, old=old)
    ref.assert_within(total, want, bound, "dtable added up")


def test_embed_of_wide_ids_is_not_cut_to_32_bits():
    table = torch.ones(4, 8, device=DEV)
    ids = torch.tensor([2**32 + 1, -2**32, 2**63 - 1, 3], device=DEV)
    assert torch.equal(sieve.embed(ids, table)[:, 0], torch.tensor([0., 0, 0, 1], device=DEV))
    got = sieve.embed_backward(torch.ones(4, 8, device=DEV), ids, 4)
    assert torch.equal(got[:, 0], torch.tensor([0., 0, 0, 1], device=DEV))


@pytest.mark.parametrize("shift", [0, 8, 3])
def test_embed_strided_rows_and_nan_of_lost_tokens(shift):
    """Rows inside wider matrices, at a 16-byte boundary or off it; what a
    token without a row holds does not matter; rows that are not part stay."""
    g = gen(shift)
    wide = randn(g, 50, 200).to(BF16)
    table = wide[:, shift:shift + 136]
    ids = torch.randint(-1, 50, (3, 100), generator=g, device=DEV)
    room = torch.full((300, 150), 7.0, device=DEV)
    out = sieve.embed(ids.flatten(), table, scale=0.5, dtype=FP32, out=room[:, shift:shift + 136])
    want, bound = ref.embed(ids.flatten(), table, 0.5, FP32)
    ref.assert_within(out, want, bound, "out")
    assert (room[:, :shift] == 7).all() and (room[:, shift + 136:] == 7).all()
    assert sieve.embed(ids, table, scale=0.5).shape == (3, 100, 136)
    dout = randn(g, 300, 150)[:, shift:shift + 136]
    dout[ids.flatten() < 0] = math.nan
    got = torch.full((50, 150), 7.0, device=DEV)
    sieve.embed_backward(dout, ids, 50, scale=0.5, out=got[:, shift:shift + 136])
    want, bound = ref.embed_backward(dout, ids, 50, 0.5, FP32)
    ref.assert_within(got[:, shift:shift + 136], want, bound, "dtable")
    assert (got[:, :shift] == 7).all() and (got[:, shift + 136:] == 7).all()


def test_embed_of_no_tokens():
    ids, table = torch.empty(0, dtype=I64, device=DEV), torch.ones(40, 24, device=DEV)
    assert sieve.embed(ids, table).shape == (0, 24)
    dout = torch.empty(0, 24, device=DEV)
    assert not sieve.embed_backward(dout, ids, 40).any()
    assert torch.equal(sieve.embed_backward(dout, ids, 40, out=table.clone(), accumulate=True), table)
    lost = torch.full((70,), -1, device=DEV)
    assert not sieve.embed_backward(torch.full((70, 24), math.nan, device=DEV), lost, 40).any()


def test_embed_refusals():
    ids, table = torch.zeros(4, dtype=I64, device=DEV), torch.ones(4, 8, device=DEV)
    d = torch.ones(4, 8, device=DEV)
    for call, what in ((lambda: sieve.embed(ids.float(), table), TypeError), (lambda: sieve.embed(ids, table.double()), TypeError),
                       (lambda: sieve.embed(ids, table.t()), ValueError), (lambda: sieve.embed(ids[::2], table), ValueError),
                       (lambda: sieve.embed(ids, table, dtype=torch.float64), TypeError),
                       (lambda: sieve.embed(ids, table, out=d[:3]), ValueError), (lambda: sieve.embed(ids, table, scale=math.inf), sieve.SieveError),
                       (lambda: sieve.embed_backward(d[:3], ids, 4), ValueError), (lambda: sieve.embed_backward(d, ids, 0), sieve.SieveError),
                       (lambda: sieve.embed_backward(d, ids, 4, accumulate=True), ValueError),
                       (lambda: sieve.embed_backward(d, ids, 4, out=d[:, :4]), ValueError)):
        with pytest.raises(what):
            call()


# ------------------------------------------------------------ residual norm
def residual_inputs(g, rows, width, dtype, wtype, pre, post, bias, gate):
    h = (randn(g, rows, width) * torch.exp(0.5 * randn(g, width)) + randn(g, width)).to(dtype)
    y = (0.5 * randn(g, rows, width) + 0.3 * randn(g, width)).to(dtype)
    kw = dict(weight=(1 + 0.3 * randn(g, width)).to(wtype) if pre else None, bias=randn(g, width).to(wtype) if pre and bias else None,
              post_weight=(1 + 0.3 * randn(g, width)).to(wtype) if post else None,
              post_bias=randn(g, width).to(wtype) if post and bias else None,
              gate={"none": lambda: None, "column": lambda: randn(g, width).to(wtype), "row": lambda: randn(g, rows, width).to(dtype)}[gate]())
    return h, y, kw


NAMES = ("dh", "dy", "dweight", "dbias", "dpost_weight", "dpost_bias", "dgate")


def check_residual(h, y, kw, alpha, rms, ds, dx):
    stream, x, stats = sieve.residual_norm(h, y, alpha=alpha, rms=rms, **kw)
    grads = sieve.residual_norm_backward(ds, dx, h, y, stats, alpha=alpha, rms=rms, **kw)
    want, bound = ref.residual_norm(h, y, **kw, alpha=alpha, rms=rms, dstream=ds, dx=dx)
    got = {k: t for k, t in dict(stream=stream, x=x, **dict(zip(NAMES, grads))).items() if t is not None}
    assert set(got) == set(want)
    for name, t in got.items():
        ref.assert_within(t, want[name], bound[name], name)
    again = sieve.residual_norm_backward(ds, dx, h, y, stats, alpha=alpha, rms=rms, **kw)
    assert all(a is b or torch.equal(a, b) for a, b in zip(grads, again))


@pytest.mark.parametrize("rows,width,dtype,wtype", [
    (1, 1, FP32, FP32), (3, 8, BF16, BF16), (23, 768, BF16, BF16), (1000, 768, BF16, FP32), (257, 256, FP16, FP16), (700, 200, FP16, FP32),
    (65, 1000, FP16, FP32), (130, 1001, FP32, FP32), (130, 1001, BF16, BF16), (300, 512, BF16, BF16), (77, 2048, FP32, FP32),
    (1300, 1024, BF16, FP32), (41, 4100, BF16, FP32), (9, 4097, FP16, FP16), (5, 8192, BF16, BF16), (330, 8192, FP32, FP32), (3, 8191, FP32, FP32),
    (2011, 33, FP32, FP32), (64, 520, BF16, BF16), (50, 1540, FP32, FP32), (50, 300, FP32, FP32),
])
@pytest.mark.parametrize("pre,post,bias,gate,rms,alpha", [
    (True, True, True, "column", False, 1.0), (True, True, False, "row", True, 0.5), (True, False, True, "none", True, 1.5),
    (False, True, True, "column", False, 1.0), (True, False, False, "column", False, -0.7), (False, True, True, "row", False, 0.0),
])
def test_residual_norm(rows, width, dtype, wtype, pre, post, bias, gate, rms, alpha):
    g = gen(rows * 7 + width)
    h, y, kw = residual_inputs(g, rows, width, dtype, wtype, pre, post, bias, gate)
    ds, dx = randn(g, rows, width).to(dtype), randn(g, rows, width).to(dtype) if pre else None
    check_residual(h, y, kw, alpha, rms, ds, dx)


def test_residual_norm_without_a_gradient_of_the_stream():
    g = gen(1)
    h, y, kw = residual_inputs(g, 40, 96, BF16, FP32, True, True, True, "column")
    check_residual(h, y, kw, 1.0, False, None, randn(g, 40, 96).to(BF16))


@pytest.mark.parametrize("shift", [0, 8, 3])
@pytest.mark.parametrize("width", [512, 1104])
def test_residual_norm_strided_and_in_place(shift, width):
    """Rows of wider matrices, the stream over h and x over y; dh over the
    stream's gradient and dy over dx."""
    g = gen(shift)
    wide = [randn(g, 60, width + 16).to(BF16) for _ in range(6)]
    h, y, gate, ds, dx, dg = (t[:, shift:shift + width] for t in wide)
    kw = dict(weight=randn(g, width).to(BF16), bias=None, post_weight=randn(g, width).to(BF16), post_bias=randn(g, width).to(BF16), gate=gate)
    want, bound = ref.residual_norm(h, y, **kw, alpha=0.9, rms=True, dstream=ds, dx=dx)
    h0, y0, rest = h.clone(), y.clone(), [t.clone() for t in wide]
    stream, x, stats = sieve.residual_norm(h, y, alpha=0.9, rms=True, out=h, x_out=y, **kw)
    assert stream is h and x is y
    ref.assert_within(h, want["stream"], bound["stream"], "stream")
    ref.assert_within(y, want["x"], bound["x"], "x")
    grads = sieve.residual_norm_backward(ds, dx, h0, y0, stats, alpha=0.9, rms=True, out=ds, dy_out=dx, **kw)
    assert grads[0] is ds and grads[1] is dx
    for name, t in zip(NAMES, grads):
        if t is not None:
            ref.assert_within(t, want[name], bound[name], name)
    for now, then in zip(wide, rest):
        assert torch.equal(now[:, :shift], then[:, :shift]) and torch.equal(now[:, shift + width:], then[:, shift + width:])


def test_residual_norm_of_no_rows_and_more_dims():
    none, w = torch.empty(0, 96, device=DEV), torch.ones(96, device=DEV)
    stream, x, stats = sieve.residual_norm(none, none, w, post_weight=w, gate=w)
    assert stream.shape == x.shape == (0, 96) and stats.shape == (4, 0)
    grads = sieve.residual_norm_backward(none, none, none, none, stats, w, post_weight=w, gate=w)
    assert all(not grads[i].any() for i in (2, 4, 6))
    g = gen(2)
    h, y = randn(g, 3, 5, 96), randn(g, 3, 5, 96)
    stream, x, stats = sieve.residual_norm(h, y, w, gate=randn(g, 3, 5, 96))
    assert stream.shape == x.shape == (3, 5, 96) and stats.shape == (4, 15)


def test_residual_norm_constant_rows():
    """No spread: the factor is 1 / sqrt(eps), the normed rows are zeros."""
    h, y, w = torch.full((4, 96), 2.5, device=DEV), torch.zeros(4, 96, device=DEV), torch.ones(96, device=DEV)
    stream, x, stats = sieve.residual_norm(h, y, w, post_weight=w)
    assert torch.equal(stream, h) and torch.equal(x, torch.zeros_like(x)) and torch.equal(stats[2], h[:, 0])


def test_residual_norm_refusals():
    h, w = torch.ones(4, 8, device=DEV), torch.ones(8, device=DEV)
    s = sieve.residual_norm(h, h, w)[2]
    for call, what in ((lambda: sieve.residual_norm(h, h), ValueError), (lambda: sieve.residual_norm(h, h, post_weight=w, bias=w), ValueError),
                       (lambda: sieve.residual_norm(h, h[:3], w), ValueError), (lambda: sieve.residual_norm(h, h.half(), w), TypeError),
                       (lambda: sieve.residual_norm(h, h, w.half()), TypeError), (lambda: sieve.residual_norm(h, h, w[:7]), ValueError),
                       (lambda: sieve.residual_norm(h.half(), h.half(), w, post_weight=w.half()), TypeError),
                       (lambda: sieve.residual_norm(h, h, w, gate=w[:7]), ValueError), (lambda: sieve.residual_norm(h, h, w, gate=h[:3]), ValueError),
                       (lambda: sieve.residual_norm(h, h, post_weight=w, x_out=h), ValueError),
                       (lambda: sieve.residual_norm(h, h, w, alpha=math.nan), sieve.SieveError),
                       (lambda: sieve.residual_norm_backward(h, None, h, h, s, w), ValueError),
                       (lambda: sieve.residual_norm_backward(None, None, h, h, s, post_weight=w), ValueError),
                       (lambda: sieve.residual_norm_backward(h, h, h, h, s[:2], w), ValueError)):
        with pytest.raises(what):
            call()


# ------------------------------------------------------------ cross entropy
def loss_inputs(g, rows, classes, width, dtype, live=1.0, bias=False, itype=I64, spread=2.0):
    weight = ((randn(g, classes, width) + 0.5 * randn(g, width)) * spread * width ** -0.5).to(dtype)
    t = torch.randint(classes, (rows,), generator=g, device=DEV)
    h = (randn(g, rows, width) + 2 * torch.rand(rows, 1, generator=g, device=DEV) * weight[t].float() * width ** 0.5 / spread).to(dtype)
    outside = torch.tensor([-1, classes, -100, 2**31 - 1], device=DEV)[torch.randint(4, (rows,), generator=g, device=DEV)]
    t = torch.where(torch.rand(rows, generator=g, device=DEV) < live, t, outside).to(itype)
    return h, weight, t, randn(g, classes) if bias else None


def check_loss(h, weight, t, bias, scale, dloss, dweight_dtype=None):
    loss, lse = sieve.cross_entropy(h, weight, t, bias=bias, scale=scale, check=True)
    dw = None if dweight_dtype is None else torch.full(weight.shape, math.nan, dtype=dweight_dtype, device=DEV)
    dh, dweight, dbias = sieve.cross_entropy_backward(dloss, h, weight, t, loss, lse, bias=bias, scale=scale, dweight=dw, check=True)
    want, bound = ref.cross_entropy(h, weight, t, bias, scale, dloss, dweight_dtype)
    for name, got in dict(loss=loss, lse=lse, dh=dh, dweight=dweight, dbias=dbias).items():
        if got is not None:
            ref.assert_within(got, want[name], bound[name], name)
    assert (dbias is None) == (bias is None)
    again = sieve.cross_entropy(h, weight, t, bias=bias, scale=scale)
    assert torch.equal(again[0], loss) and torch.equal(again[1], lse)
    again = sieve.cross_entropy_backward(dloss, h, weight, t, loss, lse, bias=bias, scale=scale, dweight=None if dw is None else dw.clone())
    assert torch.equal(again[0], dh) and torch.equal(again[1], dweight) and (bias is None or torch.equal(again[2], dbias))
    return loss, lse, dh, dweight, dbias


LOSS = [
    # rows, classes, width, type, share of rows with a target, bias, id type
    (1, 1, 8, BF16, 1.0, False, I64), (1, 2, 8, FP16, 1.0, True, I32), (5, 300, 64, BF16, 1.0, True, I64), (128, 256, 64, BF16, 1.0, False, I32),
    (129, 257, 72, FP16, 1.0, False, I64), (200, 1000, 768, BF16, 1.0, True, I64), (127, 255, 128, BF16, 0.5, True, I32),
    (1000, 4099, 256, FP16, 0.15, True, I64), (2500, 777, 136, BF16, 0.9, False, I32), (64, 20_000, 512, BF16, 1.0, True, I64),
    (3000, 513, 1032, BF16, 1.0, False, I64), (40, 130, 2048, FP16, 1.0, True, I32), (300, 33, 8, BF16, 0.3, False, I64), (700, 9001, 320, FP16, 1.0, False, I32),
    (2, 600, 16_384, BF16, 1.0, True, I64),
]


@pytest.mark.parametrize("rows,classes,width,dtype,live,bias,itype", LOSS)
@pytest.mark.parametrize("weights", ["same", "differ"])
def test_cross_entropy(rows, classes, width, dtype, live, bias, itype, weights):
    g = gen(rows + classes)
    h, weight, t, b = loss_inputs(g, rows, classes, width, dtype, live, bias, itype)
    dloss = torch.full((rows,), 8.0 / rows, device=DEV) if weights == "same" else randn(g, rows)
    check_loss(h, weight, t, b, 1.0, dloss, FP32 if rows % 2 and weights == "same" else None)


def test_cross_entropy_in_pieces_of_the_classes():
    """More scores than the workspace of the backward pass holds at a time:
    dh is added up over the pieces, the last of which ends inside a tile."""
    g = gen(13)
    h, weight, t, b = loss_inputs(g, 4_200, 140_003, 24, BF16, 0.97, True)
    check_loss(h, weight, t, b, 1.0, torch.full((4_200,), 1 / 64, device=DEV), FP32)


@pytest.mark.parametrize("scale", [20.0, 0.0, -1.5, 1e-30])
@pytest.mark.parametrize("bias", [False, True])
def test_cross_entropy_scales(scale, bias):
    g = gen(7)
    h, weight, t, b = loss_inputs(g, 333, 700, 64, BF16, 0.8, bias)
    h, weight = (x / x.float().norm(dim=1, keepdim=True) for x in (h, weight)) if scale == 20.0 else (h, weight)
    check_loss(h.to(BF16), weight.to(BF16), t, b, scale, torch.full((333,), -0.5, device=DEV))


def test_cross_entropy_rows_without_a_target_do_not_matter():
    """Whatever they hold, in h and in dloss; their results are zeros, and the
    others' are those of a call without them, bit for bit."""
    g = gen(8)
    h, weight, t, b = loss_inputs(g, 900, 500, 96, BF16, 0.6, True)
    dead = (t < 0) | (t >= 500)
    dloss = randn(g, 900)
    h[dead] = math.nan
    dloss[dead] = math.inf
    loss, lse, dh, dw, db = check_loss(h, weight, t, b, 1.0, dloss)
    assert not loss[dead].any() and not lse[dead].any() and not dh[dead].any()
    alone = sieve.cross_entropy(h[~dead], weight, t[~dead], bias=b)
    assert torch.equal(alone[0], loss[~dead]) and torch.equal(alone[1], lse[~dead])
    grads = sieve.cross_entropy_backward(dloss[~dead], h[~dead], weight, t[~dead], *alone, bias=b)
    assert torch.equal(grads[0], dh[~dead]) and torch.equal(grads[1], dw) and torch.equal(grads[2], db)


@pytest.mark.parametrize("rows", [1, 300])
def test_cross_entropy_without_any_target_or_row(rows):
    weight = torch.ones(70, 64, dtype=BF16, device=DEV)
    b = torch.zeros(70, device=DEV)
    for n in (rows, 0):
        h, t, d = torch.full((n, 64), math.nan, dtype=BF16, device=DEV), torch.full((n,), -1, device=DEV), torch.ones(n, device=DEV)
        loss, lse = sieve.cross_entropy(h, weight, t, bias=b, check=True)
        assert not loss.any() and not lse.any()
        for dt in (BF16, FP32):
            dw = torch.full((70, 64), math.nan, dtype=dt, device=DEV)
            dh, dw, db = sieve.cross_entropy_backward(d, h, weight, t, loss, lse, bias=b, dweight=dw, check=True)
            assert not dh.any() and not dw.any() and not db.any()
        kept = torch.ones(70, 64, device=DEV)
        sieve.cross_entropy_backward(d, h, weight, t, loss, lse, bias=b, dweight=kept, accumulate=True)
        assert torch.equal(kept, torch.ones_like(kept))


def test_cross_entropy_hidden_classes_and_extreme_biases():
    g = gen(9)
    h, weight, t, b = loss_inputs(g, 300, 700, 64, BF16, 1.0, True)
    b[::3] = -math.inf
    b[1::7] = -3.0e38
    t[:] = torch.where(t % 3 == 0, (t + 1) % 700, t)
    t[t % 3 == 0] = 1
    t[t % 7 == 1] = 2
    check_loss(h, weight, t, b, 1.0, torch.ones(300, device=DEV))
    # a hidden target
    t[5] = 0
    loss, lse = sieve.cross_entropy(h, weight, t, bias=b)
    assert torch.isposinf(loss[5]) and torch.isfinite(lse).all() and torch.isfinite(loss[torch.arange(300, device=DEV) != 5]).all()
    # every bias at the type's lowest: as if there were none
    low = torch.full((700,), -3.4e38, device=DEV)
    loss, lse = sieve.cross_entropy(h, weight, t, bias=low)
    assert torch.allclose(loss, torch.full_like(loss, math.log(700)), rtol=1e-5)
    # every class hidden
    loss, lse = sieve.cross_entropy(h, weight, t, bias=torch.full((700,), -math.inf, device=DEV))
    assert torch.isposinf(loss).all() and torch.isneginf(lse).all()


def test_cross_entropy_small_losses_keep_their_digits():
    """Rows that are all but certain: the loss is far below the rounding of
    the scores, and so is 1 - p in the gradient."""
    n, width = 64, 64
    h = torch.zeros(n, width, dtype=BF16, device=DEV)
    h[:, 0] = torch.arange(n, device=DEV) / 2 + 4.0
    weight = torch.zeros(3, width, dtype=BF16, device=DEV)
    weight[0, 0], weight[1, 0] = 1.0, -1.0
    t = torch.zeros(n, dtype=I64, device=DEV)
    loss, lse = sieve.cross_entropy(h, weight, t)
    x = h[:, 0].double()
    want = torch.log1p(torch.exp(-x) + torch.exp(-2 * x))
    assert ((loss.double() - want).abs() <= 2.0 ** -18 * want).all()
    check_loss(h, weight, t, None, 1.0, torch.ones(n, device=DEV))


@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_cross_entropy_takes_any_dloss(dtype):
    """Magnitudes from the type's largest to subnormal ones, zeros and both
    signs, in one call; rows whose dloss is far below the largest keep their dh."""
    g = gen(14)
    h, weight, t, b = loss_inputs(g, 640, 300, 64, dtype, 0.9, True, spread=0.5)
    exponents = torch.randint(-18, 4, (640,), generator=g, device=DEV)
    for up in (0, 80 if dtype == BF16 else 0, -100 if dtype == BF16 else 0):
        dloss = torch.where(torch.arange(640, device=DEV) % 5 == 0, 0.0, randn(g, 640)) * torch.exp2((exponents + up).float())
        check_loss(h, weight, t, b, 1.0, dloss)
    # the type's ends at once; dweight is off the type, dh is not (rows of bf16 reach as far as fp32)
    if dtype == BF16:
        dloss = torch.full((640,), 1e-42, device=DEV)
        dloss[::2] = 3e38
        loss, lse = sieve.cross_entropy(h, weight, t, bias=b)
        dh = sieve.cross_entropy_backward(dloss, h, weight, t, loss, lse, bias=b)[0]
        want, bound = ref.cross_entropy(h, weight, t, b, 1.0, dloss)
        assert want["dh"].abs().max() < 3e38
        ref.assert_within(dh, want["dh"], bound["dh"], "dh")


def test_cross_entropy_of_many_rows():
    """More rows than one list of blocks goes by, most without a target."""
    g = gen(15)
    h, weight, t, b = loss_inputs(g, 300_001, 5, 8, BF16, 0.03, True)
    check_loss(h, weight, t, b, 1.0, torch.full((300_001,), 0.25, device=DEV))


def test_cross_entropy_not_a_number_stays_in_its_row_of_dh():
    g = gen(16)
    h, weight, t, b = loss_inputs(g, 300, 700, 64, BF16)
    one = torch.ones(300, device=DEV)
    loss, lse = sieve.cross_entropy(h, weight, t)
    clean = sieve.cross_entropy_backward(one, h, weight, t, loss, lse)[0]
    h[7, 3] = math.nan
    loss, lse = sieve.cross_entropy(h, weight, t)
    dh, dw, _ = sieve.cross_entropy_backward(one, h, weight, t, loss, lse)
    rest = torch.arange(300, device=DEV) != 7
    assert dh[7].isnan().all() and torch.equal(dh[rest], clean[rest]) and dw.isnan().any()


def test_calls_that_follow_at_once_and_share_scratch():
    """Calls of different sizes one after the other on one workspace, without a
    wait between them: each one's kernels start while the ones before end, and give
    the bits they give alone."""
    g = gen(18)
    ws = sieve.Workspace()
    sizes = [(700, 3_000, 1.0), (40, 90, 0.5), (2_300, 513, 0.2), (1, 20_000, 1.0), (300, 7, 0.0)]
    inputs = [loss_inputs(g, n, v, 64, BF16, live, True) for n, v, live in sizes]

    def calls(x, workspace):
        h, weight, t, bias = x
        loss, lse = sieve.cross_entropy(h, weight, t, bias=bias, workspace=workspace)
        grads = sieve.cross_entropy_backward(torch.full_like(loss, 0.5), h, weight, t, loss, lse, bias=bias, workspace=workspace)
        table = sieve.embed_backward(grads[0], t, len(weight), workspace=workspace)
        stream, x, stats = sieve.residual_norm(h, grads[0], torch.ones(64, device=DEV))
        back = sieve.residual_norm_backward(h, grads[0], h, grads[0], stats, torch.ones(64, device=DEV), workspace=workspace)
        return (loss, lse, *grads, table, stream, x, *(t for t in back if t is not None))
    want = []
    for x in inputs:
        want.append(calls(x, None))
        torch.cuda.synchronize()
    calls(inputs[2], ws)                                 # the workspace as large as any of them needs
    for _ in range(6):
        got = [calls(x, ws) for x in inputs]
    for x, y in zip(got, want):
        assert all(torch.equal(a, b) for a, b in zip(x, y))


def test_cross_entropy_bias_gradient_alone():
    g = gen(19)
    h, weight, t, b = loss_inputs(g, 500, 900, 64, FP16, 0.7, True)
    loss, lse = sieve.cross_entropy(h, weight, t, bias=b)
    kw = dict(bias=b)
    want = sieve.cross_entropy_backward(loss, h, weight, t, loss, lse, **kw)[2]
    dh, dw, db = sieve.cross_entropy_backward(loss, h, weight, t, loss, lse, need_dh=False, need_dweight=False, check=True, **kw)
    assert dh is None and dw is None and torch.equal(db, want)


def test_cross_entropy_twice_at_once():
    """Two calls on two streams, each with its own scratch, give what they
    give alone."""
    g = gen(17)
    a, b = (loss_inputs(g, n, 3_000, 128, BF16, 0.8, True) for n in (900, 1_500))
    d = [torch.full((len(x[0]),), 0.5, device=DEV) for x in (a, b)]

    def both(x, dloss, stream=None):
        h, weight, t, bias = x
        loss, lse = sieve.cross_entropy(h, weight, t, bias=bias, stream=stream)
        return (loss, *sieve.cross_entropy_backward(dloss, h, weight, t, loss, lse, bias=bias, stream=stream))
    want = [both(x, y) for x, y in zip((a, b), d)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for i in range(2):
            got[i].append(both((a, b)[i], d[i], streams[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for res in got[i]:
            assert all(torch.equal(x, y) for x, y in zip(res, want[i]))


def test_cross_entropy_not_a_number_reaches_its_row():
    g = gen(10)
    h, weight, t, b = loss_inputs(g, 300, 700, 64, BF16)
    clean = sieve.cross_entropy(h, weight, t)
    h[7, 3] = math.nan
    loss, lse = sieve.cross_entropy(h, weight, t)
    rest = torch.arange(300, device=DEV) != 7
    assert loss[7].isnan() and lse[7].isnan() and torch.equal(loss[rest], clean[0][rest]) and torch.equal(lse[rest], clean[1][rest])


def test_cross_entropy_strides_and_parts():
    """Rows inside wider matrices; a gradient added to what is there; one
    gradient without the other gives the same bits."""
    g = gen(11)
    wide, table = randn(g, 400, 160).to(FP16), randn(g, 900, 200).to(FP16)
    h, weight = wide[:, 16:120], table[:, 8:112]
    t = torch.randint(-1, 900, (400,), generator=g, device=DEV)
    dloss = randn(g, 400)
    loss, lse = sieve.cross_entropy(h, weight, t, scale=0.1)
    old = randn(g, 900, 128)
    room = old.clone()
    kw = dict(scale=0.1)
    dh, dw, _ = sieve.cross_entropy_backward(dloss, h, weight, t, loss, lse, dweight=room[:, 8:112], accumulate=True, **kw)
    want, bound = ref.cross_entropy(h, weight, t, None, 0.1, dloss, FP32, old=old[:, 8:112])
    ref.assert_within(dh, want["dh"], bound["dh"], "dh")
    ref.assert_within(dw, want["dweight"], bound["dweight"], "dweight")
    assert torch.equal(room[:, :8], old[:, :8]) and torch.equal(room[:, 112:], old[:, 112:])
    both = sieve.cross_entropy_backward(dloss, h, weight, t, loss, lse, **kw)
    a = sieve.cross_entropy_backward(dloss, h, weight, t, loss, lse, need_dweight=False, **kw)
    b = sieve.cross_entropy_backward(dloss, h, weight, t, loss, lse, need_dh=False, **kw)
    assert a[1] is None and b[0] is None and torch.equal(a[0], both[0]) and torch.equal(b[1], both[1]) and torch.equal(dh, both[0])


def test_cross_entropy_bias_gradient_against_differences():
    """(L(b + e) - L(b - e)) / 2e for single classes: off by e^2 / 6 of the
    third derivative, at most sum |dloss| / (6 sqrt 3), and by the errors of the
    two sums of losses over 2e."""
    g = gen(12)
    h, weight, t, b = loss_inputs(g, 150, 40, 64, BF16, 0.9, True)
    dloss = torch.rand(150, generator=g, device=DEV)
    loss, lse = sieve.cross_entropy(h, weight, t, bias=b)
    dbias = sieve.cross_entropy_backward(dloss, h, weight, t, loss, lse, bias=b)[2]
    e = 2.0 ** -4
    bound = ref.cross_entropy(h, weight, t, b)[1]["loss"]
    off = e * e / 6 * float(dloss.sum()) / (6 * math.sqrt(3)) + 1.1 * float((dloss.double() * bound).sum()) / e
    for v in (0, 7, 39, int(t[t >= 0][0])):
        sums = []
        for sign in (1, -1):
            moved = b.clone()
            moved[v] += sign * e
            step = float(moved[v]) - float(b[v])
            sums.append((float((sieve.cross_entropy(h, weight, t, bias=moved)[0].double() * dloss.double()).sum()), step))
        slope = (sums[0][0] - sums[1][0]) / (sums[0][1] - sums[1][1])
        assert abs(slope - float(dbias[v])) <= off + 1e-3 * abs(float(dbias[v])), v


def test_cross_entropy_refusals():
    h, w, t = torch.ones(4, 16, dtype=BF16, device=DEV), torch.ones(9, 16, dtype=BF16, device=DEV), torch.zeros(4, dtype=I64, device=DEV)
    x = torch.ones(4, device=DEV)
    loss, lse = sieve.cross_entropy(h, w, t)
    back = lambda *a, **k: sieve.cross_entropy_backward(x, h, w, t, loss, lse, *a, **k)   # noqa: E731
    for call, what in ((lambda: sieve.cross_entropy(h.float(), w.float(), t), TypeError), (lambda: sieve.cross_entropy(h, w.half(), t), TypeError),
                       (lambda: sieve.cross_entropy(h[:, :12], w[:, :12], t), sieve.SieveError), (lambda: sieve.cross_entropy(h, w[:, :8], t), ValueError),
                       (lambda: sieve.cross_entropy(h, w, t[:3]), ValueError), (lambda: sieve.cross_entropy(h, w, t.float()), TypeError),
                       (lambda: sieve.cross_entropy(h[:, 1:9], w[:, :8], t), ValueError), (lambda: sieve.cross_entropy(h, w, t, bias=x), ValueError),
                       (lambda: sieve.cross_entropy(h, w, t, scale=math.nan), sieve.SieveError),
                       (lambda: back(dweight=torch.ones(9, 16, dtype=BF16, device=DEV), accumulate=True), ValueError),
                       (lambda: back(dweight=torch.ones(8, 16, device=DEV)), ValueError), (lambda: back(accumulate=True), ValueError),
                       (lambda: back(dweight=torch.ones(9, 16, device=DEV), need_dweight=False), ValueError),
                       (lambda: sieve.cross_entropy_backward(x[:3], h, w, t, loss, lse), ValueError)):
        with pytest.raises(what):
            call()


# ----------------------------------------------------------------- together
def training_step(ids, targets, offsets, table, p, workspaces=(None,) * 4, stream=None):
    """Token ids to the gradients of a small encoder with a tied table: embed,
    one block between its norms, cross entropy against the table."""
    heads, dim = 2, 32
    kw = dict(post_weight=p["post_w"], gate=p["gate"], weight=p["norm_w"], bias=p["norm_b"], stream=stream)
    x0 = sieve.embed(ids, table, stream=stream)
    q = x0.view(-1, heads, dim)
    o, lse_a = sieve.attention(q, q, q, offsets, workspace=workspaces[0], stream=stream)
    s, x, stats = sieve.residual_norm(x0, o.view(x0.shape), **kw)
    loss, lse = sieve.cross_entropy(x, table, targets, bias=p["out_b"], workspace=workspaces[1], stream=stream)
    dloss = torch.full_like(loss, 1 / 64)
    dtable = torch.empty(table.shape, device=table.device)
    dx, dtable, dout_b = sieve.cross_entropy_backward(dloss, x, table, targets, loss, lse, bias=p["out_b"], dweight=dtable,
                                                      workspace=workspaces[2], stream=stream)
    dh, dy, dw, db, dpw, _, dgate = sieve.residual_norm_backward(None, dx, x0, o.view(x0.shape), stats, workspace=workspaces[3], **kw)
    dq, dk, dv, _ = sieve.attention_backward(dy.view(o.shape), q, q, q, o, lse_a, offsets, workspace=workspaces[0], stream=stream)
    dx0 = dh + (dq + dk + dv).view(dh.shape)
    sieve.embed_backward(dx0, ids, table.shape[0], out=dtable, accumulate=True, workspace=workspaces[3], stream=stream)
    return dict(loss=loss, dtable=dtable, norm_w=dw, norm_b=db, post_w=dpw, gate=dgate, out_b=dout_b)


def step_inputs(seed=0, vocab=211, tokens=180):
    g = gen(seed)
    table = (0.5 * randn(g, vocab, 64)).to(BF16)
    ids = zipf(g, tokens, vocab)
    targets = torch.where(torch.rand(tokens, generator=g, device=DEV) < 0.4, torch.randint(vocab, (tokens,), generator=g, device=DEV), -1)
    offsets = torch.tensor([0, 50, 50, 121, tokens], dtype=I32, device=DEV)
    p = dict(norm_w=1 + 0.1 * randn(g, 64), norm_b=0.1 * randn(g, 64), post_w=1 + 0.1 * randn(g, 64), gate=0.5 + 0.1 * randn(g, 64),
             out_b=0.1 * randn(g, vocab))
    return ids, targets, offsets, table, p


def test_a_training_step_against_autograd():
    """The whole step against torch's autograd in 64 bits.  Between the
    operators values are rounded to bf16 (2^-8 each); ten such steps lie between the
    ids and the farthest gradient, whose roundings add up like independent
    ones: sqrt(10) 2^-8 of the norm, taken twice."""
    ids, targets, offsets, table, p = step_inputs()
    got = training_step(ids, targets, offsets, table, p)
    t64 = table.double().requires_grad_()
    leaves = {k: v.double().requires_grad_() for k, v in p.items()}
    x0 = t64[ids]
    q = x0.view(-1, 2, 32)
    parts = []
    for a, b in zip(offsets.tolist(), offsets.tolist()[1:]):
        s = torch.softmax(torch.einsum("ihd,jhd->hij", q[a:b], q[a:b]) * 32 ** -0.5, 2)
        parts.append(torch.einsum("hij,jhd->ihd", s, q[a:b]))
    y = torch.cat(parts).reshape(x0.shape)
    norm = torch.nn.functional.layer_norm
    x = norm(x0 + leaves["gate"] * norm(y, (64,), leaves["post_w"], None, 1e-5), (64,), leaves["norm_w"], leaves["norm_b"], 1e-5)
    loss = torch.nn.functional.cross_entropy(x @ t64.T + leaves["out_b"], targets, reduction="none", ignore_index=-1)
    names = list(leaves)
    want = dict(zip(["dtable"] + names, torch.autograd.grad(loss.sum() / 64, [t64] + [leaves[k] for k in names])))
    want["loss"] = loss.detach()
    for name, t in got.items():
        off = (t.double() - want[name]).norm() / want[name].norm()
        assert off < 2 * math.sqrt(10) * 2.0 ** -8, (name, float(off))


def test_a_captured_step_gives_the_same_bits_with_new_inputs():
    """Captured into a graph, replayed on other ids and targets (another
    number of rows with a target), with workspaces that are kept: the bits of
    the plain calls."""
    ids, targets, offsets, table, p = step_inputs()
    ws = tuple(sieve.Workspace() for _ in range(4))
    training_step(ids, targets, offsets, table, p, ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        training_step(ids, targets, offsets, table, p, ws)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = training_step(ids, targets, offsets, table, p, ws)
    for seed in (3, 4):
        ids2, targets2, *_ = step_inputs(seed)
        if seed == 4:
            targets2.fill_(-1)
        ids.copy_(ids2)
        targets.copy_(targets2)
        graph.replay()
        want = training_step(ids2, targets2, offsets, table, p)
        for name in out:
            assert torch.equal(out[name], want[name]), (seed, name)


def test_a_step_on_another_stream():
    ids, targets, offsets, table, p = step_inputs(5)
    want = training_step(ids, targets, offsets, table, p)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = training_step(ids, targets, offsets, table, p)
    torch.cuda.current_stream().wait_stream(s)
    for name in want:
        assert torch.equal(got[name], want[name]), name


def test_calls_with_an_explicit_stream():
    g = gen(6)
    h, weight, t, b = loss_inputs(g, 200, 300, 64, BF16, 0.7, True)
    y = randn(g, 200, 64).to(BF16)
    w = torch.ones(64, device=DEV)
    s = torch.cuda.Stream()
    want = (sieve.embed(t, weight), sieve.embed_backward(h, t, 300), *sieve.residual_norm(h, y, w),
            *sieve.cross_entropy(h, weight, t, bias=b))
    s.wait_stream(torch.cuda.current_stream())
    got = (sieve.embed(t, weight, stream=s), sieve.embed_backward(h, t, 300, stream=s), *sieve.residual_norm(h, y, w, stream=s),
           *sieve.cross_entropy(h, weight, t, bias=b, stream=s, check=True))
    s.synchronize()
    assert all(torch.equal(x, z) for x, z in zip(want, got))


# ------------------------------------------------------------------ example
def test_example_trains_on_masked_tokens():
    """The example runs, and its gradients are those of torch's autograd in 64
    bits on the same weights: some 25 roundings to bf16 (2^-8 each) lie between the
    ids and the farthest gradient and add up like independent ones, 5 * 2^-8 of the
    norm, taken twice."""
    import os
    import sys
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import train_masked_tokens as example
    got = example.main(["--docs", "300", "--vocab", "2000", "--steps", "2"])
    assert torch.allclose(got["rows"].norm(dim=1), torch.ones(300, device=DEV), atol=1e-5) and len(got["losses"]) == 2
    model = example.Encoder(150, torch.device(DEV), seed=3)
    ids, offsets = example.documents(9, 150, torch.device(DEV), seed=4)
    hidden, targets = example.masked(ids, 0.3, seed=5)
    loss, grads = model.loss_and_grads(hidden, targets, offsets)
    p = {k: (v.bfloat16() if k.startswith("w_") or k == "table" else v).double().requires_grad_() for k, v in model.p.items()}
    width, heads, dim, reach = example.WIDTH, example.HEADS, example.DIM, example.REACH

    def rms(x, w):
        return x / (x.square().mean(1, keepdim=True) + 1e-5).sqrt() * w
    h0 = p["table"][hidden] * math.sqrt(width)
    x0 = torch.nn.functional.layer_norm(h0, (width,), p["norm0"])
    q, k, v = (x0 @ p["w_qkv"]).view(-1, 3, heads, dim).unbind(1)
    parts = []
    for a, b in zip(offsets.tolist(), offsets.tolist()[1:]):
        place = torch.arange(b - a, device=DEV)
        at = model.buckets.long()[(place[None] - place[:, None]).clamp(-reach, reach) + reach]
        s = torch.einsum("ihd,jhd->hij", q[a:b], k[a:b]) * dim ** -0.5 + p["rel"][at].permute(2, 0, 1)
        parts.append(torch.einsum("hij,jhd->ihd", torch.softmax(s, 2), v[a:b]))
    h1 = h0 + p["gate0"] * rms(torch.cat(parts).reshape(-1, heads * dim) @ p["w_o"], p["post0"])
    y1 = torch.relu(rms(h1, p["norm1"]) @ p["w_up"]) @ p["w_down"]
    x2 = rms(h1 + p["gate1"] * rms(y1, p["post1"]), p["norm2"])
    want = torch.nn.functional.cross_entropy(x2 @ p["table"].T + p["out_bias"], targets, ignore_index=-1)
    assert abs(float(loss) - float(want.detach())) < 2.0 ** -6 * float(want.detach())
    for name, t in zip(p, torch.autograd.grad(want, list(p.values()))):
        off = float((grads[name].double() - t).norm() / t.norm())
        assert off < 10 * 2.0 ** -8, (name, off)
