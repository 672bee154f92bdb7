"""Arguments of the encoder operators at the edges of what they take, on the
GPU against their definitions in 64 bits (encoder_reference)."""
import pytest
import torch

import encoder_reference as ref
import paper_2608_03199_gb300 as sieve
from test_gpu_encoder import BF16, DEV, FP16, FP32, attention_inputs, check_attention, gen, randn  # noqa: F401

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
