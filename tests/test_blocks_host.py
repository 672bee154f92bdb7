"""What of the operators around an encoder's blocks needs no GPU: the
library's refusals and workspace sizes, the binding's, and the reference that
the GPU tests use."""
import ctypes as C
import math

import pytest
import torch

import blocks_reference as ref
import encoder_reference
import paper_2608_03199_gb300 as sieve
from paper_2608_03199_gb300.blocks import (CrossEntropyArgsC, CrossEntropyGradsC, ResidualNormArgsC,
                                           ResidualNormGradsC)

P, ODD, BIG = C.c_void_p(256), C.c_void_p(258), 1 << 40


def embed(ids=P, idt=3, tokens=7, table=P, ts=64, vocab=10, width=64, tdt=0, scale=1.0, out=P, os=64, dt=0):
    return sieve.lib().sieve_embed(ids, idt, tokens, table, ts, vocab, width, tdt, scale, out, os, dt, None)


@pytest.mark.parametrize("bad", [
    dict(ids=None), dict(ids=ODD), dict(ids=C.c_void_p(260), idt=4), dict(idt=2), dict(tokens=-1), dict(tokens=(1 << 30) + 1),
    dict(table=None), dict(table=ODD), dict(ts=63), dict(vocab=0), dict(vocab=(1 << 26) + 1), dict(width=0), dict(width=16385),
    dict(tdt=3), dict(scale=math.nan), dict(scale=math.inf), dict(out=None), dict(out=ODD), dict(os=63), dict(dt=-1)])
def test_embed_refuses(bad):
    assert embed(**bad) == -1


def embed_backward(dout=P, ds=64, ids=P, idt=3, tokens=7, vocab=10, width=64, dt=0, scale=1.0, dtable=P, gs=64, gdt=0, acc=0,
                   ws=P, have=BIG):
    return sieve.lib().sieve_embed_backward(dout, ds, ids, idt, tokens, vocab, width, dt, scale, dtable, gs, gdt, acc, ws, have,
                                            None)


@pytest.mark.parametrize("bad", [
    dict(dout=None), dict(dout=ODD), dict(ds=60), dict(ids=None), dict(idt=0), dict(tokens=-1), dict(vocab=0), dict(width=0),
    dict(dt=9), dict(scale=math.inf), dict(dtable=None), dict(dtable=ODD), dict(gs=1), dict(gdt=4), dict(acc=2), dict(acc=-1)])
def test_embed_backward_refuses(bad):
    assert embed_backward(**bad) == -1
    n = C.c_size_t()
    lib = sieve.lib()
    assert lib.sieve_embed_backward_workspace_size(1000, 50, 64, C.byref(n)) == 0 and n.value > 1000 * 8
    assert lib.sieve_embed_backward_workspace_size(1000, 50, 64, None) == -1
    assert embed_backward(have=0) == -3 and embed_backward(ws=None) == -3 and embed_backward(ws=C.c_void_p(264)) == -3


def norm_args(**kw):
    base = dict(rows=5, width=64, dtype=2, weight_dtype=2, alpha=1.0, eps=1e-5, h=256, y=256, h_stride=64, y_stride=64, weight=256,
                bias=256, post_weight=256, post_bias=256, gate_kind=1, gate=256)
    return ResidualNormArgsC(**{**base, **kw})


def norm_grads(**kw):
    base = dict(dstream=256, dx=256, dstream_stride=64, dx_stride=64, stats=256, dh=256, dy=256, dgate=256, dh_stride=64, dy_stride=64,
                dgate_stride=64, dweight=256, dbias=256, dpost_weight=256, dpost_bias=256)
    return ResidualNormGradsC(**{**base, **kw})


@pytest.mark.parametrize("bad", [
    dict(rows=-1), dict(width=0), dict(width=8193), dict(dtype=3), dict(weight_dtype=1), dict(rms=2), dict(alpha=math.nan),
    dict(alpha=math.inf), dict(eps=-1e-5), dict(eps=math.inf), dict(weight=None, bias=None, post_weight=None, post_bias=None),
    dict(weight=None), dict(post_weight=None), dict(h=None), dict(y=None), dict(h=257), dict(h_stride=63), dict(y_stride=0),
    dict(weight=257), dict(post_bias=257), dict(gate_kind=0), dict(gate=None), dict(gate=257), dict(gate_kind=3),
    dict(gate_kind=2, gate_stride=63)])
def test_residual_norm_refuses(bad):
    lib, a = sieve.lib(), C.byref(norm_args(**bad))
    assert lib.sieve_residual_norm(a, P, 64, P, 64, P, None) == -1
    assert lib.sieve_residual_norm_backward(a, C.byref(norm_grads()), P, BIG, None) == -1


def test_residual_norm_refuses_results():
    lib, a = sieve.lib(), C.byref(norm_args())
    odd = C.c_void_p(257)
    for s, ss, x, xs, st in ((None, 64, P, 64, P), (P, 63, P, 64, P), (P, 64, None, 64, P), (P, 64, P, 1, P), (P, 64, P, 64, ODD),
                             (odd, 64, P, 64, P)):
        assert lib.sieve_residual_norm(a, s, ss, x, xs, st, None) == -1
    last = C.byref(norm_args(weight=None, bias=None))
    assert lib.sieve_residual_norm(last, P, 64, P, 64, P, None) == -1          # x without a weight
    assert lib.sieve_residual_norm(None, P, 64, P, 64, P, None) == -1
    for bad in (dict(dx=None), dict(dx_stride=3), dict(dstream_stride=3), dict(stats=None), dict(stats=258), dict(dh=None), dict(dy=None),
                dict(dy=257), dict(dgate=None), dict(dgate=257), dict(dweight=None), dict(dbias=None), dict(dpost_bias=None),
                dict(dpost_weight=257)):
        assert lib.sieve_residual_norm_backward(a, C.byref(norm_grads(**bad)), P, BIG, None) == -1, bad
    assert lib.sieve_residual_norm_backward(a, None, P, BIG, None) == -1
    assert lib.sieve_residual_norm_backward(last, C.byref(norm_grads(dx=None, dstream=None, dweight=None, dbias=None)), P, BIG, None) == -1
    assert lib.sieve_residual_norm_backward(a, C.byref(norm_grads()), P, 0, None) == -3
    n = C.c_size_t()
    assert lib.sieve_residual_norm_backward_workspace_size(100, 64, C.byref(n)) == 0 and n.value > 0
    assert lib.sieve_residual_norm_backward_workspace_size(100, 8193, C.byref(n)) == -1


def loss_args(**kw):
    base = dict(rows=5, classes=100, width=64, dtype=2, target_type=4, scale=1.0, h=256, weight=256, h_stride=64, weight_stride=64,
                bias=256, targets=256)
    return CrossEntropyArgsC(**{**base, **kw})


def loss_grads(**kw):
    base = dict(dloss=256, loss=256, lse=256, dh=256, dweight=256, dh_stride=64, dweight_stride=64, dweight_dtype=2, dbias=256)
    return CrossEntropyGradsC(**{**base, **kw})


@pytest.mark.parametrize("bad", [
    dict(rows=-1), dict(rows=(1 << 24) + 1), dict(classes=0), dict(classes=(1 << 24) + 1), dict(width=0), dict(width=60),
    dict(width=16392), dict(dtype=0), dict(dtype=3), dict(target_type=2), dict(scale=math.nan), dict(scale=math.inf)])
def test_cross_entropy_refuses_sizes(bad):
    lib, n = sieve.lib(), C.c_size_t()
    for size in (lib.sieve_cross_entropy_workspace_size, lib.sieve_cross_entropy_backward_workspace_size):
        assert size(C.byref(loss_args()), C.byref(n)) == 0 and n.value >= 256
        assert size(C.byref(loss_args(**bad)), C.byref(n)) == -1
        assert size(None, C.byref(n)) == -1 and size(C.byref(loss_args()), None) == -1
    assert lib.sieve_cross_entropy(C.byref(loss_args(**bad)), P, P, P, BIG, None) == -1
    assert lib.sieve_cross_entropy_backward(C.byref(loss_args(**bad)), C.byref(loss_grads()), P, BIG, None) == -1


@pytest.mark.parametrize("bad", [
    dict(h=None), dict(h=264), dict(h_stride=60), dict(h_stride=56), dict(h_stride=-64), dict(weight=None), dict(weight=8),
    dict(weight_stride=0), dict(weight_stride=68), dict(bias=258), dict(targets=None), dict(targets=260)])
def test_cross_entropy_refuses_pointers(bad):
    lib = sieve.lib()
    assert lib.sieve_cross_entropy(C.byref(loss_args(**bad)), P, P, P, BIG, None) == -1
    assert lib.sieve_cross_entropy_backward(C.byref(loss_args(**bad)), C.byref(loss_grads()), P, BIG, None) == -1


def test_cross_entropy_refuses_results():
    lib, a = sieve.lib(), C.byref(loss_args())
    for loss, lse in ((None, P), (P, None), (ODD, P), (P, ODD)):
        assert lib.sieve_cross_entropy(a, loss, lse, P, BIG, None) == -1
    assert lib.sieve_cross_entropy(a, P, P, P, 0, None) == -3
    assert lib.sieve_cross_entropy(a, P, P, C.c_void_p(264), BIG, None) == -3
    for bad in (dict(dloss=None), dict(loss=None), dict(lse=258), dict(dh=264), dict(dh_stride=60), dict(dweight=264),
                dict(dweight_stride=60), dict(dweight_dtype=1), dict(accumulate=1), dict(accumulate=2, dweight_dtype=0),
                dict(dbias=258)):
        assert lib.sieve_cross_entropy_backward(a, C.byref(loss_grads(**bad)), P, BIG, None) == -1, bad
    assert lib.sieve_cross_entropy_backward(C.byref(loss_args(bias=None)), C.byref(loss_grads()), P, BIG, None) == -1
    assert lib.sieve_cross_entropy_backward(a, None, P, BIG, None) == -1
    assert lib.sieve_cross_entropy_backward(a, C.byref(loss_grads()), P, 0, None) == -3


def test_cross_entropy_workspaces_hold_no_scores():
    """Far below the scores of a large call: pieces of the classes, and parts
    of the statistics."""
    n = C.c_size_t()
    a = loss_args(rows=65_536, classes=262_144, width=64, bias=None)
    assert sieve.lib().sieve_cross_entropy_workspace_size(C.byref(a), C.byref(n)) == 0 and n.value < 2 * 65_536 * 262_144 // 30
    assert sieve.lib().sieve_cross_entropy_backward_workspace_size(C.byref(a), C.byref(n)) == 0 and n.value < 2 * 65_536 * 262_144 // 16


def test_cpu_tensors_are_refused():
    x, t = torch.randn(3, 8), torch.zeros(3, dtype=torch.int64)
    for call in (lambda: sieve.embed(t, x), lambda: sieve.embed_backward(x, t, 5), lambda: sieve.residual_norm(x, x, x[0]),
                 lambda: sieve.cross_entropy(x.half(), x.half(), t)):
        with pytest.raises(TypeError):
            call()


def close(got, want, name):
    assert torch.allclose(got, want, rtol=1e-9, atol=1e-11), name


@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("pre,post,bias,gate", [(True, True, True, "column"), (True, True, False, "row"), (True, False, True, "column"),
                                                (False, True, True, "row"), (True, False, False, "none"), (False, True, False, "column")])
def test_reference_residual_norm_agrees_with_autograd(rms, pre, post, bias, gate):
    encoder_reference.U[torch.float64], encoder_reference.TINY[torch.float64] = 2.0 ** -53, 1e-300
    g = torch.Generator().manual_seed(3)
    n, width = 7, 12

    def leaf(*shape):
        return torch.randn(*shape, generator=g).double().requires_grad_()

    h, y = leaf(n, width), leaf(n, width)
    kw = dict(weight=leaf(width) if pre else None, bias=leaf(width) if pre and bias else None,
              post_weight=leaf(width) if post else None, post_bias=leaf(width) if post and bias else None,
              gate=None if gate == "none" else leaf(width) if gate == "column" else leaf(n, width))

    def norm(v, w, b):
        if rms:
            out = torch.nn.functional.rms_norm(v, (width,), w, 1e-5)
            return out if b is None else out + b
        return torch.nn.functional.layer_norm(v, (width,), w, b, 1e-5)

    u = norm(y, kw["post_weight"], kw["post_bias"]) if post else y
    s = 0.7 * h + (u if kw["gate"] is None else kw["gate"] * u)
    outs = [s] + ([norm(s, kw["weight"], kw["bias"])] if pre else [])
    ds, dx = (torch.randn(n, width, generator=g).double() for _ in range(2))
    names = ["dh", "dy"] + ["d" + k for k, t in kw.items() if t is not None]
    want = torch.autograd.grad(outs, [h, y] + [t for t in kw.values() if t is not None], [ds, dx][:len(outs)])
    plain = {k: None if t is None else t.detach() for k, t in kw.items()}
    res, _ = ref.residual_norm(h.detach(), y.detach(), **plain, alpha=0.7, rms=rms, dstream=ds, dx=dx if pre else None)
    close(res["stream"], s.detach(), "stream")
    if pre:
        close(res["x"], outs[1].detach(), "x")
    for name, t in zip(names, want):
        close(res[name], t, name)


def test_reference_cross_entropy_agrees_with_autograd_and_differences():
    encoder_reference.U[torch.float64], encoder_reference.TINY[torch.float64] = 2.0 ** -53, 1e-300
    g = torch.Generator().manual_seed(4)
    h, w, b = (torch.randn(*s, generator=g).double().requires_grad_() for s in ((6, 8), (11, 8), (11,)))
    t = torch.tensor([3, -1, 0, 10, 11, 3])
    dloss = torch.randn(6, generator=g).double()
    loss = torch.nn.functional.cross_entropy(1.5 * h @ w.T + b, torch.where(t > 10, -1, t), reduction="none", ignore_index=-1)
    want = torch.autograd.grad(loss, (h, w, b), dloss)
    res, _ = ref.cross_entropy(h.detach(), w.detach(), t, b.detach(), 1.5, dloss)
    close(res["loss"], loss.detach(), "loss")
    for name, x in zip(("dh", "dweight", "dbias"), want):
        close(res[name], x, name)
    step = torch.randn(11, 8, generator=g).double()
    up, down = (ref.cross_entropy(h.detach(), w.detach() + e * step, t, b.detach(), 1.5)[0]["loss"] @ dloss for e in (1e-5, -1e-5))
    assert abs((up - down) / 2e-5 - (res["dweight"] * step).sum()) < 1e-7


def test_reference_embed_agrees_with_autograd():
    table = torch.randn(5, 6, dtype=torch.float64, requires_grad=True)
    encoder_reference.U[torch.float64], encoder_reference.TINY[torch.float64] = 2.0 ** -53, 1e-300
    ids = torch.tensor([[4, 0, 4], [-1, 2, 5]])
    out, _ = ref.embed(ids, table.detach(), 1.5, torch.float64)
    real = (ids >= 0) & (ids < 5)
    plain = torch.where(real[..., None], 1.5 * table[ids.clamp(0, 4)], 0.0)
    close(out, plain.detach(), "out")
    dout = torch.randn(2, 3, 6).double()
    close(ref.embed_backward(dout, ids, 5, 1.5, torch.float64)[0], torch.autograd.grad(plain, table, dout)[0], "dtable")
