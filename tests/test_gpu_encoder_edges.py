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
