"""Arguments of the encoder operators at the edges of what they take, on the
GPU against their definitions in 64 bits (encoder_reference)."""
import pytest
import torch

import encoder_reference as ref
import paper_2608_03199_gb300 as sieve
from test_gpu_encoder import BF16, DEV, FP16, attention_inputs, check_attention

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


SCALES = [0.0, -0.0, 1e-42, -0.3]


@pytest.mark.parametrize("scale", SCALES)
@pytest.mark.parametrize("dim,dtype,buckets,causal", [(64, BF16, 0, False), (64, FP16, 0, True), (128, BF16, 0, True), (40, BF16, 32, False)])
def test_attention_takes_any_finite_scale(dim, dtype, buckets, causal, scale):
    """Zero (a mean over the keys seen), less than a normal number, negative:
    with and without a table, documents that end inside a tile."""
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
