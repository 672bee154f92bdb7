"""The encoder operators on the GPU against their definitions in 64 bits
(encoder_reference): layer norm, attention over packed documents with a
relative position bias, unit pooling, and their backward passes."""
import math

import pytest
import torch

import encoder_reference as ref
import paper_2608_03199_gb300 as sieve

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32


def gen(seed):
    return torch.Generator(DEV).manual_seed(seed)


def randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


# --------------------------------------------------------------------- norm
@pytest.mark.parametrize("rows,width,dtype,wtype,bias", [
    (1, 1, FP32, FP32, True), (3, 8, BF16, BF16, True), (23, 768, BF16, BF16, True), (1000, 768, BF16, FP32, True),
    (257, 256, FP16, FP16, False), (65, 1000, FP16, FP32, True), (130, 1001, FP32, FP32, False),
    (130, 1001, BF16, BF16, True), (77, 2048, FP32, FP32, True), (41, 4100, BF16, FP32, True),
    (9, 4097, FP16, FP16, True), (5, 16384, BF16, BF16, True), (5, 16384, FP32, FP32, True), (3, 16383, FP32, FP32, True),
    (20011, 33, FP32, FP32, True), (5000, 512, BF16, FP32, True), (2, 130, FP32, FP32, True), (611, 4096, FP16, FP32, False),
])
def test_layer_norm(rows, width, dtype, wtype, bias):
    g = gen(rows * 7 + width)
    x = (randn(g, rows, width) * torch.exp(randn(g, width)) + 2 * randn(g, width)).to(dtype)
    w, b = (1 + 0.3 * randn(g, width)).to(wtype), randn(g, width).to(wtype) if bias else None
    dy = randn(g, rows, width).to(dtype)
    y, mean, rstd = sieve.layer_norm(x, w, b, eps=1e-5)
    dx, dw, db = sieve.layer_norm_backward(dy, x, w, mean, rstd, need_dbias=bias)
    assert y.dtype == dx.dtype == dtype and dw.dtype == wtype
    want, bound = ref.layer_norm(x, w, b, 1e-5, dy)
    for name, got in dict(y=y, dx=dx, dw=dw, **({"db": db} if bias else {})).items():
        ref.assert_within(got, want[name], bound[name], name)
    again = sieve.layer_norm_backward(dy, x, w, mean, rstd, need_dbias=bias)
    assert torch.equal(again[0], dx) and torch.equal(again[1], dw)


@pytest.mark.parametrize("shift", [0, 8, 3])
def test_layer_norm_strided_rows_and_in_place(shift):
    """Rows of a wider matrix at a 16-byte boundary or off it; dx over dy, y over x."""
    g = gen(shift)
    wide = randn(g, 50, 800).to(BF16)
    x = wide[:, shift:shift + 512]
    w = randn(g, 512).to(BF16)
    want, bound = ref.layer_norm(x, w, None, 1e-6, x)
    kept = x.clone()
    y, mean, rstd = sieve.layer_norm(x, w, eps=1e-6, out=x)
    assert y is x
    ref.assert_within(x, want["y"], bound["y"], "y")
    assert torch.equal(wide[:, shift + 512:], wide[:, shift + 512:].clone())
    dy = kept.clone()
    dx, dw, db = sieve.layer_norm_backward(dy, kept, w, mean, rstd, out=dy)
    assert dx is dy
    ref.assert_within(dx, want["dx"], bound["dx"], "dx")
    ref.assert_within(dw, want["dw"], bound["dw"], "dw")


def test_layer_norm_large_mean_constant_rows_and_no_rows():
    g = gen(5)
    x = 3000 + randn(g, 64, 768)
    w = torch.ones(768, device=DEV)
    y, mean, rstd = sieve.layer_norm(x, w)
    want, bound = ref.layer_norm(x, w, None, 1e-5)
    ref.assert_within(y, want["y"], bound["y"], "y")
    flat = torch.full((4, 96), 2.5, device=DEV)
    y, mean, rstd = sieve.layer_norm(flat, torch.ones(96, device=DEV), eps=1e-5)
    assert torch.equal(y, torch.zeros_like(y)) and torch.equal(mean, flat[:, 0])
    none = torch.empty(0, 96, device=DEV)
    y, mean, rstd = sieve.layer_norm(none, torch.ones(96, device=DEV))
    dx, dw, db = sieve.layer_norm_backward(none, none, torch.ones(96, device=DEV), mean, rstd)
    assert y.shape == none.shape and not dw.any() and not db.any() and dw.shape == (96,)


def test_layer_norm_nonfinite_rows_stay_apart():
    g = gen(6)
    x = randn(g, 9, 300)
    x[3, 7], x[5, 0] = math.nan, math.inf
    w = torch.ones(300, device=DEV)
    y, _, _ = sieve.layer_norm(x, w)
    bad = torch.tensor([3, 5], device=DEV)
    assert y[bad].isnan().any(1).all()
    keep = torch.ones(9, dtype=torch.bool, device=DEV)
    keep[bad] = False
    assert y[keep].isfinite().all()


# ---------------------------------------------------------------- attention
def attention_inputs(seed, qlen, klen, heads, kv_heads, dim, dtype, buckets, reach, causal, fused=False):
    g = gen(seed)
    nq, nk = sum(qlen), sum(klen)
    if fused:
        assert qlen == klen
        whole = randn(g, nq, heads + 2 * kv_heads, dim).to(dtype)
        q, k, v = whole[:, :heads], whole[:, heads:heads + kv_heads], whole[:, heads + kv_heads:]
    else:
        q, k, v = (randn(g, n, h, dim).to(dtype) for n, h in ((nq, heads), (nk, kv_heads), (nk, kv_heads)))
    dout = randn(g, nq, heads, dim).to(dtype)
    table = randn(g, buckets, heads) if buckets else None
    bmap = sieve.relative_buckets(buckets, reach, bidirectional=not causal, device=DEV) if buckets else None
    return q, k, v, dout, table, bmap


def check_attention(q, k, v, dout, qlen, klen, table=None, buckets=None, causal=False, scale=None, backward=True):
    off, qoff = ref.offsets_of(klen, DEV), ref.offsets_of(qlen, DEV)
    kw = dict(q_offsets=None if qlen == klen else qoff, table=table, buckets=buckets, causal=causal, scale=scale)
    out, lse = sieve.attention(q, k, v, off, check=True, **kw)
    want, bound = ref.attention(q, k, v, qlen, klen, table, buckets, causal, scale, dout if backward else None)
    ref.assert_within(out, want["out"], bound["out"], "out")
    ref.assert_within(lse, want["lse"], bound["lse"], "lse")
    if not backward:
        return out, lse
    dq, dk, dv, dtable = sieve.attention_backward(dout, q, k, v, out, lse, off, check=True, **kw)
    for name, got in (("dq", dq), ("dk", dk), ("dv", dv), ("dtable", dtable)):
        if got is not None:
            ref.assert_within(got, want[name], bound[name], name)
    return out, lse, dq, dk, dv, dtable


LENGTHS = {
    "one": [1], "short": [23], "edge": [127, 0, 128, 129, 1], "ragged": [300, 0, 0, 17, 511, 64, 1, 260],
    "long": [1500], "empty": [0, 0], "many": [3] * 70 + [0] * 5 + [140],
}


@pytest.mark.parametrize("lengths", sorted(LENGTHS))
@pytest.mark.parametrize("heads,kv_heads,dim,dtype,buckets,reach,causal", [
    (3, 3, 64, BF16, 32, 128, False), (4, 2, 64, FP16, 0, 0, True), (4, 1, 128, BF16, 32, 128, True),
    (2, 2, 128, FP16, 0, 0, False), (6, 2, 40, BF16, 16, 64, False), (2, 1, 96, BF16, 64, 256, True),
    (1, 1, 8, FP16, 4, 2, False), (2, 2, 32, BF16, 64, 256, False),
])
def test_attention_of_documents(lengths, heads, kv_heads, dim, dtype, buckets, reach, causal):
    n = LENGTHS[lengths]
    q, k, v, dout, table, bmap = attention_inputs(len(n) + dim, n, n, heads, kv_heads, dim, dtype, buckets, reach, causal)
    check_attention(q, k, v, dout, n, n, table, bmap, causal)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dim", [64, 128])
def test_attention_between_lengths_and_rows_that_see_nothing(causal, dim):
    """Queries and keys of different lengths: more queries than keys leaves
    the first ones of a causal document without a key, a document without
    keys leaves all of its queries without one."""
    qlen, klen = [5, 300, 130, 7, 0, 40, 1], [400, 129, 0, 7, 9, 3, 260]
    q, k, v, dout, table, bmap = attention_inputs(3, qlen, klen, 4, 2, dim, BF16, 32, 128, causal)
    out, lse, dq, dk, dv, dtable = check_attention(q, k, v, dout, qlen, klen, table, bmap, causal)
    first = sum(qlen[:2])
    assert not out[first:first + 130].any() and torch.isneginf(lse[:, first:first + 130]).all()
    assert not dq[first:first + 130].any()
    gone = sum(klen[:4])
    assert not dk[gone:gone + 9].any() and not dv[gone:gone + 9].any()


@pytest.mark.parametrize("new", [1, 3, 16, 70])
@pytest.mark.parametrize("heads,kv_heads,dim,dtype,buckets", [(8, 2, 128, BF16, 32), (4, 4, 64, FP16, 0), (3, 1, 72, BF16, 16)])
def test_attention_of_new_tokens(new, heads, kv_heads, dim, dtype, buckets):
    """The next tokens of growing documents, from none kept to thousands."""
    klen = [5000, 0, 1, 2, 16, 129, 777, 128]
    qlen = [new] * len(klen)
    q, k, v, dout, table, bmap = attention_inputs(new, qlen, klen, heads, kv_heads, dim, dtype, buckets, 64, True)
    off = ref.offsets_of(klen, DEV)
    kw = dict(table=table, buckets=bmap, causal=True)
    q4, d4 = q.view(len(klen), new, heads, dim), dout.view(len(klen), new, heads, dim)
    out, lse = sieve.attention(q4, k, v, off, check=True, **kw)
    want, bound = ref.attention(q, k, v, qlen, klen, table, bmap, True, None, dout)
    ref.assert_within(out.view(q.shape), want["out"], bound["out"], "out")
    ref.assert_within(lse, want["lse"], bound["lse"], "lse")
    again, lse2 = sieve.attention(q4, k, v, off, **kw)
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    dq, dk, dv, dtable = sieve.attention_backward(d4, q4, k, v, out, lse, off, check=True, **kw)
    for name, got in (("dq", dq.view(q.shape)), ("dk", dk), ("dv", dv), ("dtable", dtable)):
        if got is not None:
            ref.assert_within(got, want[name], bound[name], name)


@pytest.mark.parametrize("same,causal", [(True, False), (False, True)])
def test_attention_of_thousands_of_documents(same, causal):
    """More documents than a block keeps in view at a time, with long runs of
    empty ones, and heads that make every block start over."""
    klen = [i * 7 % 5 for i in range(1100)] + [0] * 1200 + [130] + [0] * 70 + [1, 2, 3] * 100 + [0] * 40
    qlen = klen if same else klen[::-1]
    q, k, v, dout, table, bmap = attention_inputs(11, qlen, klen, 3, 3, 16, BF16, 16, 20, causal)
    check_attention(q, k, v, dout, qlen, klen, table, bmap, causal)


def test_attention_of_one_new_token_over_one_long_document():
    klen = [40_001]
    q, k, v, _, table, bmap = attention_inputs(9, [1], klen, 4, 1, 128, BF16, 32, 128, True)
    out, lse = sieve.attention(q[None], k, v, ref.offsets_of(klen, DEV), table=table, buckets=bmap, causal=True, check=True)
    want, bound = ref.attention(q, k, v, [1], klen, table, bmap, True)
    ref.assert_within(out[0], want["out"], bound["out"], "out")
    ref.assert_within(lse, want["lse"], bound["lse"], "lse")


@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_other_documents_and_rows_past_the_last_do_not_matter(value):
    """NaN and infinities in the neighbouring documents and in rows that
    belong to no document leave a document's results as they are, bit for bit."""
    n = [100, 37, 200]
    q, k, v, dout, table, bmap = attention_inputs(1, n, n, 2, 1, 64, BF16, 32, 128, False)
    pad = torch.full((50, 2, 64), value, dtype=BF16, device=DEV)
    off = ref.offsets_of(n, DEV)
    kw = dict(table=table, buckets=bmap)
    out, lse = sieve.attention(q, k, v, off, **kw)
    grads = sieve.attention_backward(dout, q, k, v, out, lse, off, **kw)
    mid = slice(100, 137)
    bad = []
    for t in (q, k, v, dout):
        t = torch.cat([t, pad[:, :t.shape[1]]])
        kept = t[mid].clone()
        t[:] = value
        t[mid] = kept
        bad.append(t)
    q2, k2, v2, d2 = bad
    out2, lse2 = sieve.attention(q2, k2, v2, off, **kw)
    assert torch.equal(out2[mid], out[mid]) and torch.equal(lse2[:, mid], lse[:, mid])
    grads2 = sieve.attention_backward(d2, q2, k2, v2, out2, lse2, off, **kw)
    for a, b in zip(grads[:3], grads2[:3]):
        assert torch.equal(a[mid], b[mid])
    one = sieve.attention(q2[None, 136:137].expand(3, 1, 2, 64).contiguous(), k2, v2, off, **kw)[0]
    want = sieve.attention(q[None, 136:137].expand(3, 1, 2, 64).contiguous(), k, v, off, **kw)[0]
    assert torch.equal(one[1], want[1])


def test_hidden_buckets_and_lowest_values():
    """A bias of -inf hides a bucket (all of them: zeros and -inf); the
    type's lowest value does not: where nothing else is seen it counts."""
    n = [200, 3]
    q, k, v, dout, table, bmap = attention_inputs(2, n, n, 2, 2, 64, BF16, 32, 128, False)
    table[20:, 0] = -math.inf
    table[:, 1] = -math.inf
    out, lse, dq, dk, dv, dtable = check_attention(q, k, v, dout, n, n, table, bmap)
    assert not out[:, 1].any() and torch.isneginf(lse[1]).all() and not dq[:, 1].any() and not dv[:, 1].any()
    table[:] = torch.finfo(FP32).min
    out, lse = sieve.attention(q, k, v, ref.offsets_of(n, DEV), table=table, buckets=bmap)
    mean = torch.cat([v[:200].double().mean(0, keepdim=True).expand(200, -1, -1),
                      v[200:].double().mean(0, keepdim=True).expand(3, -1, -1)])
    bound = 3 * ref.U[BF16] * torch.cat([v[:200].double().abs().mean(0, keepdim=True).expand(200, -1, -1),
                                         v[200:].double().abs().mean(0, keepdim=True).expand(3, -1, -1)])
    ref.assert_within(out, mean, bound, "out")


@pytest.mark.parametrize("causal", [False, True])
def test_parts_of_one_projection_and_strided_gradients(causal):
    n = [129, 64, 300]
    heads, kv_heads, dim = 4, 2, 64
    q, k, v, dout, table, bmap = attention_inputs(4, n, n, heads, kv_heads, dim, FP16, 32, 128, causal, fused=True)
    off = ref.offsets_of(n, DEV)
    kw = dict(table=table, buckets=bmap, causal=causal)
    out, lse = sieve.attention(q, k, v, off, **kw)
    plain = sieve.attention(q.contiguous(), k.contiguous(), v.contiguous(), off, **kw)
    assert torch.equal(out, plain[0]) and torch.equal(lse, plain[1])
    want = sieve.attention_backward(dout, q.contiguous(), k.contiguous(), v.contiguous(), out, lse, off, **kw)
    whole = torch.full((sum(n), heads + 2 * kv_heads + 1, dim), 7.0, dtype=FP16, device=DEV)
    parts = (whole[:, :heads], whole[:, heads:heads + kv_heads], whole[:, heads + kv_heads:-1])
    got = sieve.attention_backward(dout, q, k, v, out, lse, off, grads=parts, **kw)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    assert bool((whole[:, -1] == 7).all())
    # heads before tokens
    qh, kh, vh = (t.transpose(0, 1).contiguous().transpose(0, 1) for t in (q, k, v))
    assert torch.equal(sieve.attention(qh, kh, vh, off, **kw)[0], out)


def test_attention_gradient_against_differences():
    """Central differences of the 64-bit forward along random directions."""
    n = [40, 0, 150]
    q, k, v, dout, table, bmap = attention_inputs(8, n, n, 4, 2, 64, FP16, 16, 64, False)
    off = ref.offsets_of(n, DEV)
    out, lse = sieve.attention(q, k, v, off, table=table, buckets=bmap)
    grads = sieve.attention_backward(dout, q, k, v, out, lse, off, table=table, buckets=bmap)
    _, bound = ref.attention(q, k, v, n, n, table, bmap, dout=dout)
    g = gen(80)
    base = [t.double() for t in (q, k, v, table)]
    for i, name in enumerate(("dq", "dk", "dv", "dtable")):
        way = randn(g, *base[i].shape).double()
        eps = 1e-4
        sides = []
        for sign in (1, -1):
            moved = list(base)
            moved[i] = base[i] + sign * eps * way
            # the reference takes its bounds' unit roundoff from the type it is given
            o = _forward64(*moved, n, bmap)
            sides.append((o * dout.double()).sum())
        slope = (sides[0] - sides[1]) / (2 * eps)
        # differences: eps^2 of the third derivative, far below the bounds' sum
        room = (bound[name] * way.abs()).sum() + 1e-6 * slope.abs()
        assert (slope - (grads[i].double() * way).sum()).abs() <= room, name


def _forward64(q, k, v, table, lengths, bmap):
    out = torch.zeros_like(q)
    share = q.shape[1] // k.shape[1]
    reach = bmap.shape[0] // 2
    s0 = 0
    for n in lengths:
        s = slice(s0, s0 + n)
        s0 += n
        if not n:
            continue
        pos = torch.arange(n, device=DEV)
        at = bmap.long()[(pos[None] - pos[:, None]).clamp(-reach, reach) + reach]
        for h in range(q.shape[1]):
            score = q[s, h] @ k[s, h // share].T * q.shape[2] ** -0.5 + table[at, h]
            out[s, h] = torch.softmax(score, 1) @ v[s, h // share]
    return out


def test_attention_gradient_is_the_same_each_time():
    n = [700, 90, 300]
    q, k, v, dout, table, bmap = attention_inputs(12, n, n, 4, 2, 64, BF16, 32, 128, False)
    off = ref.offsets_of(n, DEV)
    kw = dict(table=table, buckets=bmap)
    out, lse = sieve.attention(q, k, v, off, **kw)
    a = sieve.attention_backward(dout, q, k, v, out, lse, off, **kw)
    b = sieve.attention_backward(dout, q, k, v, out, lse, off, **kw)
    assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_long_cache_past_32_bit_offsets():
    """Tokens whose elements lie more than 2^31 apart from the first."""
    tokens, heads, dim = 300_000, 64, 128
    cache = torch.zeros(tokens, heads, dim, dtype=BF16, device=DEV)
    g = gen(3)
    cache[-300:] = randn(g, 300, heads, dim).to(BF16)
    assert cache.numel() > 1 << 31
    klen = [tokens - 300, 300]
    q = randn(g, 2, 1, heads, dim).to(BF16)
    out, lse = sieve.attention(q, cache, cache, ref.offsets_of(klen, DEV), causal=True, check=True)
    want, bound = ref.attention(q[1], cache[-300:], cache[-300:], [1], [300], causal=True)
    ref.assert_within(out[1], want["out"], bound["out"], "out")
    assert not out[0].any()
    ref.assert_within(lse[:, :1], torch.full_like(lse[:, :1], math.log(klen[0])).double(),
                      torch.full((heads, 1), 1e-4, device=DEV).double(), "lse")


def test_another_stream_and_side_by_side_calls():
    n = [400, 30]
    q, k, v, dout, table, bmap = attention_inputs(13, n, n, 4, 2, 64, BF16, 32, 128, False)
    off = ref.offsets_of(n, DEV)
    want = sieve.attention(q, k, v, off, table=table, buckets=bmap)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    results = [sieve.attention(q, k, v, off, table=table, buckets=bmap, stream=s) for s in streams for _ in range(4)]
    torch.cuda.synchronize()
    assert all(torch.equal(o, want[0]) and torch.equal(x, want[1]) for o, x in results)


# --------------------------------------------------------------------- pool
@pytest.mark.parametrize("lengths,width,dtype", [
    ([1], 1, FP32), ([0, 3, 0], 96, BF16), ([128, 129, 1, 0, 500], 768, BF16), ([4096], 256, FP32), ([7] * 300, 33, FP16),
    ([1000, 2], 1024, FP16), ([50, 60], 4100, BF16), ([130], 16384, FP32), ([0], 64, FP32), ([300, 5], 1001, BF16),
])
def test_unit_pool(lengths, width, dtype):
    g = gen(width)
    h = (randn(g, sum(lengths), width) + randn(g, width)).to(dtype)
    drows = randn(g, len(lengths), width)
    off = ref.offsets_of(lengths, DEV)
    rows, norms = sieve.unit_pool(h, off)
    dh = sieve.unit_pool_backward(drows, rows, norms, off, h.shape[0], dtype=dtype)
    want, bound = ref.unit_pool(h, lengths, drows if sum(lengths) else None)
    ref.assert_within(rows, want["rows"], bound["rows"], "rows")
    if sum(lengths):
        ref.assert_within(dh, want["dh"], bound["dh"], "dh")
    assert torch.equal(sieve.unit_pool(h, off)[0], rows)


@pytest.mark.parametrize("size", [1e-38, 1e-25, 1e25, 1e37])
def test_unit_pool_of_means_whose_squares_leave_fp32(size):
    h = randn(gen(5), 70, 96)
    off = ref.offsets_of([3, 0, 67], DEV)
    rows, norms = sieve.unit_pool(h, off)
    small, small_norms = sieve.unit_pool(h * size, off)
    # h * size rounds every element by half an ulp (subnormals, at 1e-38, by
    # 2^-150: 1e-7 of the size), and so does every step of the sums
    means = torch.stack([h[:3].mean(0), h[:1].mean(0) * 0, h[3:].mean(0)])
    spread = h.abs().max() / means.norm(dim=1).clamp(min=1e-3)
    bound = (80 * 2.0 ** -23 * spread)[:, None]
    assert ((small - rows).abs() <= bound).all()
    assert ((small_norms.double() / size - norms.double()).abs() <= bound[:, 0] * norms).all()


def test_unit_pool_strided_rows_zero_means_and_other_documents():
    g = gen(77)
    wide = randn(g, 300, 900).to(BF16)
    lengths = [100, 37, 160]
    off = ref.offsets_of(lengths, DEV)
    for shift in (0, 8, 1):
        h = wide[:, shift:shift + 512]
        rows, norms = sieve.unit_pool(h, off)
        want, bound = ref.unit_pool(h[:297], lengths)
        ref.assert_within(rows, want["rows"], bound["rows"], "rows")
    bad = wide.clone()
    bad[:100], bad[137:] = math.nan, math.inf
    assert torch.equal(sieve.unit_pool(bad[:, :512], off)[0][1], sieve.unit_pool(wide[:, :512], off)[0][1])
    opposite = torch.stack([wide[0], -wide[0]]).contiguous()
    rows, norms = sieve.unit_pool(opposite, ref.offsets_of([2], DEV))
    assert not rows.any() and not norms.any()
    assert not sieve.unit_pool_backward(torch.ones_like(rows), rows, norms, ref.offsets_of([2], DEV), 2).any()


# ----------------------------------------------------------------- refusals
def test_refusals():
    x = torch.randn(4, 64, device=DEV)
    w = torch.ones(64, device=DEV)
    for bad, kind in ((dict(weight=w[:32]), ValueError), (dict(weight=w.half()), TypeError), (dict(x=x.cpu()), TypeError),
                      (dict(x=x.double()), TypeError), (dict(bias=w[::2]), ValueError), (dict(x=x.t()), ValueError),
                      (dict(eps=-1.0), sieve.SieveError), (dict(eps=math.nan), sieve.SieveError)):
        with pytest.raises(kind):
            sieve.layer_norm(**{**dict(x=x, weight=w), **bad})
    with pytest.raises(sieve.SieveError):
        sieve.layer_norm(torch.randn(2, 16385, device=DEV), torch.ones(16385, device=DEV))
    n = [5, 6]
    q, k, v, dout, table, bmap = attention_inputs(1, n, n, 4, 2, 64, BF16, 32, 128, False)
    ok = dict(q=q, k=k, v=v, offsets=ref.offsets_of(n, DEV), table=table, buckets=bmap)
    sieve.attention(**ok)
    for bad, kind in ((dict(q=q.float(), k=k.float(), v=v.float()), TypeError), (dict(k=k.half()), TypeError),
                      (dict(k=k[:5]), ValueError), (dict(q=q[:, :3]), ValueError), (dict(buckets=None), ValueError),
                      (dict(table=table[:, :2]), ValueError), (dict(table=table.half()), TypeError),
                      (dict(offsets=ok["offsets"].long()), TypeError), (dict(buckets=bmap[:-1]), ValueError),
                      (dict(scale=math.inf), sieve.SieveError), (dict(q=q[:5]), ValueError),
                      (dict(table=torch.zeros(65, 4, device=DEV)), sieve.SieveError),
                      (dict(q=q[..., :60], k=k[..., :60], v=v[..., :60]), sieve.SieveError),
                      (dict(out=torch.empty_like(q).transpose(0, 1).contiguous().transpose(0, 1)), ValueError)):
        with pytest.raises(kind):
            sieve.attention(**{**ok, **bad})
    wide = torch.zeros(11, 2, 136, dtype=BF16, device=DEV)
    with pytest.raises(sieve.SieveError):
        sieve.attention(wide, wide, wide, ok["offsets"])
    off_by_one = torch.zeros(11 * 4 * 64 + 1, dtype=BF16, device=DEV)[1:].view(11, 4, 64)
    with pytest.raises(sieve.SieveError):
        sieve.attention(**{**ok, "q": off_by_one})
    out, lse = sieve.attention(**ok)
    with pytest.raises(ValueError):
        sieve.attention_backward(dout, q, k, v, out, lse[:, :4], ok["offsets"])
    with pytest.raises(TypeError):
        sieve.attention_backward(dout.float(), q, k, v, out, lse, ok["offsets"])
    with pytest.raises(ValueError):
        sieve.unit_pool(torch.randn(3, 4, 5, device=DEV), ok["offsets"])
    with pytest.raises(TypeError):
        sieve.unit_pool(torch.randn(11, 5, device=DEV), ok["offsets"].long())


# ------------------------------------------------------------------ example
def test_example_runs_the_operators_together():
    """The example's documents come out of the encoder as unit rows, almost
    all planted copies are found, and gradient steps lower the loss."""
    import os
    import sys
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import encode_and_deduplicate as example
    got = example.main(["--docs", "1500", "--train", "3"])
    assert torch.allclose(got["rows"].norm(dim=1), torch.ones(1500, device=DEV), atol=1e-5)
    assert got["found"] > 0.9
    assert got["losses"][-1] < got["losses"][0]
