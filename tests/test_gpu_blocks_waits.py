"""The cross entropy's bounded device waits give up cleanly (failure detection
without a GPU fault).  ``wait_limit`` shortens the one for a tile's products, in
the warps that have no copies or products of their own in flight; with a limit
of one poll it runs out (a tile takes far longer), the kernel lets what it
issued land, frees its tensor memory and returns, the status word says
SIEVE_ETIMEOUT, and the same context and workspace then give the usual bits."""
import ctypes as C

import pytest
import torch

import paper_2608_03199_gb300 as sieve
from test_blocks_host import BIG, P, loss_args, loss_grads
from test_gpu_blocks import loss_inputs
from test_gpu_encoder import BF16, DEV, FP16, FP32, gen

ETIMEOUT = -7


@pytest.mark.gpu
@pytest.mark.parametrize("rows,classes,width,dtype,live,bias", [(700, 9_001, 320, BF16, 1.0, False), (4_000, 2_000, 768, FP16, 0.8, True), (60, 300, 64, BF16, 1.0, True)])
def test_cross_entropy_wait_gives_up_and_the_context_survives(rows, classes, width, dtype, live, bias):
    g = gen(rows)
    h, weight, t, b = loss_inputs(g, rows, classes, width, dtype, live, bias)
    dloss = torch.rand(rows, generator=g, device=DEV)
    loss, lse = sieve.cross_entropy(h, weight, t, bias=b, check=True)
    want = (loss, lse, *sieve.cross_entropy_backward(dloss, h, weight, t, loss, lse, bias=b, check=True))
    ws = sieve.Workspace()

    def forward(limit):
        return sieve.cross_entropy(h, weight, t, bias=b, workspace=ws, check=True, wait_limit=limit)

    def backward(limit, **kw):
        return sieve.cross_entropy_backward(dloss, h, weight, t, loss, lse, bias=b, workspace=ws, check=True, wait_limit=limit, **kw)
    for call in (forward, backward, lambda limit: backward(limit, dweight=torch.zeros(weight.shape, dtype=FP32, device=DEV), accumulate=True)):
        with pytest.raises(sieve.SieveError) as e:
            call(1)
        assert e.value.status == ETIMEOUT
        got = (*forward(0), *backward(1 << 30))
        assert all(x is y or torch.equal(x, y) for x, y in zip(got, want))


@pytest.mark.gpu
def test_cross_entropy_status_is_read_back_later():
    g = gen(3)
    h, weight, t, _ = loss_inputs(g, 700, 3_000, 256, BF16)
    ws = sieve.Workspace()
    sieve.cross_entropy(h, weight, t, workspace=ws, wait_limit=1)
    assert sieve.encoder_status(ws, None) == ETIMEOUT
    sieve.cross_entropy(h, weight, t, workspace=ws)
    assert sieve.encoder_status(ws, None) == 0


def test_cross_entropy_refuses_a_negative_limit():
    a, n, lib = C.byref(loss_args(wait_limit=-1)), C.c_size_t(), sieve.lib()
    assert lib.sieve_cross_entropy_workspace_size(a, C.byref(n)) == -1
    assert lib.sieve_cross_entropy(a, P, P, P, BIG, None) == -1
    assert lib.sieve_cross_entropy_backward(a, C.byref(loss_grads()), P, BIG, None) == -1
