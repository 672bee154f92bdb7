"""Arguments of the encoder operators at the edges of what they take, on the
GPU against their definitions in 64 bits (encoder_reference)."""
import ctypes as C
import threading

import pytest
import torch

import encoder_reference as ref
import paper_2608_03199_gb300 as sieve
from paper_2608_03199_gb300.encoder import AttentionArgsC
from test_gpu_encoder import BF16, DEV, FP16, FP32, attention_inputs, check_attention, gen, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim,dtype,buckets,causal", [(128, BF16, 0, False), (128, FP16, 32, True), (96, BF16, 16, False),
                                                      (64, BF16, 32, True)])
def test_attention_of_many_documents_of_one_tile(dim, dtype, buckets, causal):
    """Work of one step after another, where a block runs ahead of its slowest
    warp the furthest: every work's row statistics must still reach it."""
    n = [1 + i * 37 % 128 for i in range(700)]
    q, k, v, dout, table, bmap = attention_inputs(21 + dim, n, n, 4, 2, dim, dtype, buckets, 64, causal)
    check_attention(q, k, v, dout, n, n, table, bmap, causal)


@pytest.mark.parametrize("new", [0, 1, 3])
@pytest.mark.parametrize("buckets", [0, 32])
def test_attention_over_no_keys_at_all(new, buckets):
    """Queries of documents that hold no key yet: zeros, -inf, zero gradients."""
    qlen, klen = [new or 130] * 3, [0, 0, 0]
    q, k, v, dout, table, bmap = attention_inputs(31, qlen, klen, 4, 2, 64, BF16, buckets, 64, True)
    off = ref.offsets_of(klen, DEV)
    kw = dict(table=table, buckets=bmap, causal=True, check=True)
    if new:
        q, dout = q.view(3, new, 4, 64), dout.view(3, new, 4, 64)
    else:
        kw["q_offsets"] = ref.offsets_of(qlen, DEV)
    out, lse = sieve.attention(q, k, v, off, **kw)
    assert not out.any() and torch.isneginf(lse).all()
    dq, dk, dv, dtable = sieve.attention_backward(dout, q, k, v, out, lse, off, **kw)
    assert not dq.any() and dk.shape == k.shape and dv.shape == v.shape
    assert dtable is None or not dtable.any()


SCALES = [0.0, -0.0, 1e-42, -0.3, 1.0]


@pytest.mark.parametrize("scale", SCALES)
@pytest.mark.parametrize("dim,dtype,buckets,causal", [(64, BF16, 0, False), (64, FP16, 0, True), (128, BF16, 0, True), (40, BF16, 32, False)])
def test_attention_takes_any_finite_scale(dim, dtype, buckets, causal, scale):
    """Zero (a mean over the keys seen), less than a normal number, negative,
    and one: with and without a table, documents that end inside a tile."""
    qlen, klen = ([200, 0, 33, 128, 5], [200, 0, 33, 128, 5]) if dim != 128 else ([200, 7, 33, 130, 5], [129, 0, 300, 128, 3])
    q, k, v, dout, table, bmap = attention_inputs(41, qlen, klen, 4, 2, dim, dtype, buckets, 64, causal)
    check_attention(q, k, v, dout, qlen, klen, table, bmap, causal, scale)


def check_new_tokens(new, klen, heads, kv_heads, dim, dtype, buckets, causal, scale=None, seed=0):
    """Forward and backward of `new` tokens for each document."""
    qlen = [new] * len(klen)
    q, k, v, dout, table, bmap = attention_inputs(seed + new, qlen, klen, heads, kv_heads, dim, dtype, buckets, 64, causal)
    off, shape = ref.offsets_of(klen, DEV), (len(klen), new, heads, dim)
    kw = dict(table=table, buckets=bmap, causal=causal, scale=scale, check=True)
    out, lse = sieve.attention(q.view(shape), k, v, off, **kw)
    grads = sieve.attention_backward(dout.view(shape), q.view(shape), k, v, out, lse, off, **kw)
    want, bound = ref.attention(q, k, v, qlen, klen, table, bmap, causal, scale, dout)
    for name, got in zip(("out", "lse", "dq", "dk", "dv", "dtable"), (out, lse, *grads)):
        if got is not None:
            ref.assert_within(got.reshape(want[name].shape), want[name], bound[name], name)


@pytest.mark.parametrize("scale", SCALES)
@pytest.mark.parametrize("buckets,causal", [(0, True), (0, False), (32, True)])
def test_attention_of_new_tokens_takes_any_finite_scale(buckets, causal, scale):
    check_new_tokens(3, [700, 0, 1, 2, 129, 640], 6, 2, 64, BF16, buckets, causal, scale)


@pytest.mark.parametrize("new", [128, 129, 300])
@pytest.mark.parametrize("heads,kv_heads,dim,dtype,buckets,causal", [(4, 2, 64, BF16, 32, True), (3, 1, 128, FP16, 0, True),
                                                                     (2, 2, 72, BF16, 16, False)])
def test_attention_of_many_new_tokens(new, heads, kv_heads, dim, dtype, buckets, causal):
    """A tile of new tokens for each document, one more, and several tiles,
    over fewer and over more kept tokens."""
    check_new_tokens(new, [500, 0, 1, 128, 299, 130], heads, kv_heads, dim, dtype, buckets, causal)


@pytest.mark.parametrize("left", [0, 8, 3])
def test_layer_norm_in_place_leaves_the_columns_beside_it(left):
    """y over x and dx over dy inside a wider matrix: the columns on both sides stay."""
    g = gen(left)
    wide, wide_dy = randn(g, 50, 800).to(BF16), randn(g, 50, 800).to(BF16)
    kept, kept_dy = wide.clone(), wide_dy.clone()
    part = slice(left, left + 512)
    w = randn(g, 512).to(BF16)
    want, bound = ref.layer_norm(kept[:, part], w, None, 1e-6, kept_dy[:, part])
    y, mean, rstd = sieve.layer_norm(wide[:, part], w, eps=1e-6, out=wide[:, part])
    ref.assert_within(y, want["y"], bound["y"], "y")
    dx, dw, _ = sieve.layer_norm_backward(wide_dy[:, part], kept[:, part], w, mean, rstd, out=wide_dy[:, part])
    ref.assert_within(dx, want["dx"], bound["dx"], "dx")
    for now, before in ((wide, kept), (wide_dy, kept_dy)):
        assert torch.equal(now[:, :left], before[:, :left]) and torch.equal(now[:, left + 512:], before[:, left + 512:])


def test_every_call_on_another_stream_and_with_a_kept_workspace():
    """Bit for bit what the current stream and scratch of their own give."""
    g = gen(81)
    n = [300, 0, 90]
    off = ref.offsets_of(n, DEV)
    q, k, v, dout, table, bmap = attention_inputs(82, n, n, 4, 2, 64, BF16, 32, 64, True)
    h, w, drows = randn(g, sum(n), 256), randn(g, 256), randn(g, 3, 256)

    def calls(**kw):
        plain = {key: x for key, x in kw.items() if key != "workspace"}
        y, mean, rstd = sieve.layer_norm(h, w, **plain)
        dx, dw, db = sieve.layer_norm_backward(y, h, w, mean, rstd, **kw)
        out, lse = sieve.attention(q, k, v, off, table=table, buckets=bmap, causal=True, check=True, **kw)
        grads = sieve.attention_backward(dout, q, k, v, out, lse, off, table=table, buckets=bmap, causal=True, check=True, **kw)
        rows, norms = sieve.unit_pool(h, off, **kw)
        dh = sieve.unit_pool_backward(drows, rows, norms, off, h.shape[0], **plain)
        return (y, mean, rstd, dx, dw, db, out, lse, *grads, rows, norms, dh)

    want = calls()
    torch.cuda.synchronize()
    s, ws = torch.cuda.Stream(), sieve.Workspace()
    for _ in range(3):
        for got in (calls(stream=s), calls(workspace=ws), calls(stream=s, workspace=sieve.Workspace())):
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_attention_from_a_new_host_thread():
    """A thread that has made no CUDA call yet has no current context."""
    n = [60, 5]
    q, k, v, dout, table, bmap = attention_inputs(72, n, n, 2, 1, 64, BF16, 32, 64, False)
    off, s = ref.offsets_of(n, DEV), torch.cuda.current_stream().cuda_stream
    want = sieve.attention(q, k, v, off, table=table, buckets=bmap)
    out, lse = torch.empty_like(q), torch.empty_like(want[1])
    ws = torch.empty(1 << 16, dtype=torch.uint8, device=DEV)
    a = AttentionArgsC(2, 2, 1, 64, 2, 65, 65, 0, 0, 0.125, 32, 64, 0, None, off.data_ptr(), q.data_ptr(), k.data_ptr(),
                       v.data_ptr(), 128, 64, 64, 64, 64, 64, table.data_ptr(), bmap.data_ptr())
    rc = []
    t = threading.Thread(target=lambda: rc.append(sieve.lib().sieve_attention(
        C.byref(a), out.data_ptr(), lse.data_ptr(), ws.data_ptr(), ws.numel(), s)))
    t.start()
    t.join()
    assert rc == [0]
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


def test_host_threads_with_tables_of_different_reach():
    """A kernel's shared-memory limit belongs to the process: calls with small
    tables must not lower it under a launch with large ones."""
    n, lib, strides = [150, 40], sieve.lib(), (C.c_int64 * 6)(128, 64, 64, 64, 64, 64)
    jobs = []
    for reach in (64, 256, 8, 200):
        q, k, v, dout, table, bmap = attention_inputs(71, n, n, 2, 1, 64, BF16, 16, reach, False)
        off, s = ref.offsets_of(n, DEV), torch.cuda.Stream()
        out, lse = sieve.attention(q, k, v, off, table=table, buckets=bmap)
        got = [torch.zeros_like(t) for t in (out, lse, q, k, v, table)]
        want = (out, lse, *sieve.attention_backward(dout, q, k, v, out, lse, off, table=table, buckets=bmap))
        ws = torch.empty(1 << 20, dtype=torch.uint8, device=DEV)
        a = AttentionArgsC(2, 2, 1, 64, 2, 190, 190, 0, 0, 0.125, 16, reach, 0, None, off.data_ptr(), q.data_ptr(), k.data_ptr(),
                           v.data_ptr(), 128, 64, 64, 64, 64, 64, table.data_ptr(), bmap.data_ptr())
        jobs.append((a, [t.data_ptr() for t in got], dout.data_ptr(), ws, s, got, want, (q, k, v, table, bmap, off, dout)))
    torch.cuda.synchronize()
    codes = []

    def work(a, p, dout, ws, s, *kept):
        for _ in range(1500):
            rc = lib.sieve_attention(C.byref(a), p[0], p[1], ws.data_ptr(), ws.numel(), s.cuda_stream)
            rc = rc or lib.sieve_attention_backward(C.byref(a), dout, p[0], p[1], p[2], p[3], p[4], strides, p[5],
                                                    ws.data_ptr(), ws.numel(), s.cuda_stream)
            if rc:
                codes.append((rc, lib.sieve_last_cuda_error()))
                return

    threads = [threading.Thread(target=work, args=j) for j in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not codes, codes
    for *_, got, want, _ in jobs:
        assert all(torch.equal(x, y) for x, y in zip(got, want))


LOWEST = torch.finfo(FP32).min


@pytest.mark.parametrize("value", [LOWEST, -LOWEST, -1e30, 1e30])
@pytest.mark.parametrize("dim,dtype,causal", [(64, BF16, False), (64, FP16, True), (128, FP16, False), (96, BF16, True)])
def test_biases_beside_which_scores_vanish(dim, dtype, causal, value):
    """Biases so large that adding the score changes nothing, in 64 bits
    either: the keys that carry the row's largest share its weight evenly, and
    the gradients follow.  One head all of that value; one where it stands at
    the near buckets alone, so that some rows see nothing else; one without."""
    n = [200, 1, 0, 2, 130]
    q, k, v, dout, table, bmap = attention_inputs(51, n, n, 3, 3, dim, dtype, 32, 64, causal)
    table[:, 0] = value
    table[bmap[64 - 2:64 + 3].long().unique(), 1] = value
    out, lse, dq, dk, dv, dtable = check_attention(q, k, v, dout, n, n, table, bmap, causal)
    assert lse[:2].isfinite().logical_or(lse[:2] == -torch.inf).all()
    off = ref.offsets_of(n, DEV)
    again = sieve.attention_backward(dout, q, k, v, out, lse, off, table=table, buckets=bmap, causal=causal)
    assert all(torch.equal(a, b) for a, b in zip(again, (dq, dk, dv, dtable)))


@pytest.mark.parametrize("value", [LOWEST, -1e30])
def test_new_tokens_with_biases_beside_which_scores_vanish(value):
    klen = [300, 0, 1, 129]
    qlen = [3] * 4
    q, k, v, dout, table, bmap = attention_inputs(52, qlen, klen, 4, 2, 64, BF16, 32, 64, True)
    table[:, 1] = value
    off, kw = ref.offsets_of(klen, DEV), dict(table=table, buckets=bmap, causal=True, check=True)
    out, lse = sieve.attention(q.view(4, 3, 4, 64), k, v, off, **kw)
    grads = sieve.attention_backward(dout.view(4, 3, 4, 64), q.view(4, 3, 4, 64), k, v, out, lse, off, **kw)
    want, bound = ref.attention(q, k, v, qlen, klen, table, bmap, True, None, dout)
    for name, got in zip(("out", "lse", "dq", "dk", "dv", "dtable"), (out, lse, *grads)):
        ref.assert_within(got.reshape(want[name].shape), want[name], bound[name], name)


@pytest.mark.parametrize("value", [-3e4, -1e6, -1e9, -1e30, LOWEST, 1e6, 1e9])
def test_probabilities_of_a_row_add_up_to_one_under_any_bias(value):
    """With dout = 1 every column of dv adds up to the number of queries.  In
    fp16 P is off by 2^-11, dv by as much again; a score that rounds to another
    fp32 neighbour in the two passes moves single P, not their sum's 2^-10."""
    n = [200, 130]
    q, k, v, dout, table, bmap = attention_inputs(53, n, n, 2, 1, 64, FP16, 32, 64, False)
    table += value if value > LOWEST / 2 else 0
    if value <= LOWEST / 2:
        table[:] = value
    off, kw = ref.offsets_of(n, DEV), dict(table=table, buckets=bmap, check=True)
    out, lse = sieve.attention(q, k, v, off, **kw)
    dv = sieve.attention_backward(torch.ones_like(dout), q, k, v, out, lse, off, **kw)[2]
    for a, b in ((0, 200), (200, 330)):
        total = dv[a:b].double().sum(0) / (2 * (b - a))        # two heads share the key head
        assert ((total - 1).abs() <= 2 * ref.U[FP16] + 2.0 ** -10).all(), float(total.mean())


def test_status_of_a_call_without_work():
    """A call that launches nothing leaves the status word of a call that went well."""
    lib, off = sieve.lib(), torch.zeros(3, dtype=torch.int32, device=DEV)
    t = torch.zeros(64, dtype=BF16, device=DEV)
    a = AttentionArgsC(dtype=2, heads=1, kv_heads=1, head_dim=64, nseq=2, scale=1.0, k_offsets=off.data_ptr(), q=t.data_ptr(),
                       k=t.data_ptr(), v=t.data_ptr(), q_token_stride=64, q_head_stride=64, k_token_stride=64,
                       k_head_stride=64, v_token_stride=64, v_head_stride=64)
    stream = torch.cuda.current_stream().cuda_stream
    strides = (C.c_int64 * 6)(*[64] * 6)
    p = t.data_ptr()
    for call in (lambda ws: lib.sieve_attention(C.byref(a), p, p, ws.data_ptr(), ws.numel(), stream),
                 lambda ws: lib.sieve_attention_backward(C.byref(a), p, p, p, p, p, p, strides, None, ws.data_ptr(),
                                                         ws.numel(), stream)):
        ws = torch.full((1 << 16,), 0xFF, dtype=torch.uint8, device=DEV)
        assert call(ws) == 0
        assert sieve.encoder_status(ws, stream) == 0


def test_unit_pool_gradient_of_the_smallest_means():
    """A mean below 2^-128 has no reciprocal in fp32; a document whose rows
    get no gradient has none all the same, and others what fp32 can hold."""
    h = torch.zeros(4, 96, device=DEV)
    h[:, 0] = 1e-39
    off = ref.offsets_of([3, 1], DEV)
    rows, norms = sieve.unit_pool(h, off)
    drows = torch.zeros(2, 96, device=DEV)
    drows[1, 1] = 0.125
    dh = sieve.unit_pool_backward(drows, rows, norms, off, 4)
    want = torch.zeros(4, 96, device=DEV, dtype=torch.float64)
    want[3, 1] = 0.125 / norms[1].double()
    ref.assert_within(dh, want, 2.0 ** -21 * want, "dh")


@pytest.mark.parametrize("size", [1e-5, 1e-4, 1.0])
@pytest.mark.parametrize("dim,buckets,causal", [(64, 0, False), (64, 32, True), (128, 0, True), (128, 32, False)])
def test_fp16_gradients_of_long_documents(dim, buckets, causal, size):
    """The probabilities of thousands of keys are small, and dS smaller by
    dout: in fp16 it must not round among the subnormals."""
    n = [2000, 3, 150]
    q, k, v, dout, table, bmap = attention_inputs(91, n, n, 2, 1, dim, FP16, buckets, 64, causal)
    dout[1000:1500] = 0         # rows without a gradient beside rows with one
    check_attention(q, k, v, dout * size, n, n, table, bmap, causal)


def test_fp16_gradients_whose_ds_leaves_the_type():
    """dS past 65,504 with dq and dk far below it."""
    n = [2] * 60 + [3] * 40 + [5, 40]
    q, k, v, dout, *_ = attention_inputs(92, n, n, 4, 2, 64, FP16, 0, 0, False)
    check_attention(q * 0.01, k * 0.01, v * 30, dout * 600, n, n)


def test_fp16_weights_far_below_the_largest():
    """The key at a query's own place carries nearly all of its row, every
    other 2^-20 of that: their weights must not round among fp16's subnormals
    (the early queries meet the large one first)."""
    n = 3000
    table = torch.zeros(4, 1, device=DEV)
    table[1] = 14.0                                             # no distance
    bmap = torch.tensor([0, 1, 0], dtype=torch.int32, device=DEV)
    v = 0.5 + randn(gen(95), n, 1, 64).abs()
    v[:100] = 0                                                 # rows made of the small weights alone
    q = torch.zeros(n, 1, 64, dtype=FP16, device=DEV)
    check_attention(q, q, v.to(FP16), None, [n], [n], table, bmap, backward=False)


@pytest.mark.parametrize("new", [0, 1])
def test_lse_of_even_weights_is_the_logarithm_of_their_number(new):
    """With q = 0 a row's sum is the number of its keys, exactly, so lse is off
    by the logarithm's own ulp, its conversion from base 2 and one rounding."""
    klen = [1, 2, 3, 5, 100, 1000, 3001, 7777, 20_000]
    qlen = [new] * len(klen) if new else [min(b, 5) for b in klen]
    k = randn(gen(61), sum(klen), 1, 64).to(BF16)
    off = ref.offsets_of(klen, DEV)
    if new:
        lse = sieve.attention(k.new_zeros(len(klen), 1, 1, 64), k, k, off)[1]
    else:
        lse = sieve.attention(k.new_zeros(sum(qlen), 1, 64), k, k, off, q_offsets=ref.offsets_of(qlen, DEV))[1]
    want = torch.tensor([b for a, b in zip(qlen, klen) for _ in range(a)], device=DEV).double().log()[None]
    ref.assert_within(lse, want, 2.0 ** -22 * want, "lse")
