"""What of the encoder operators needs no GPU: the bucket map, the library's
refusals and workspace sizes, and the reference the GPU tests use."""
import ctypes as C
import math

import pytest
import torch

import encoder_reference as ref
import paper_2608_03199_gb300 as sieve
from paper_2608_03199_gb300.encoder import AttentionArgsC


@pytest.mark.parametrize("buckets,reach,both", [(32, 128, True), (32, 128, False), (16, 64, True), (64, 256, False), (4, 2, True),
                                                (2, 2, False)])
def test_bucket_map(buckets, reach, both):
    """The map equals the logarithmic rule, evaluated in 64 bits with room
    for distances whose quotient of logarithms is a whole number."""
    m = sieve.relative_buckets(buckets, reach, bidirectional=both, device="cpu")
    assert m.dtype == torch.int32 and m.shape == (2 * reach + 1,) and int(m.min()) >= 0 and int(m.max()) < buckets
    half = buckets // 2 if both else buckets
    near = half // 2
    for dist in range(-reach, reach + 1):
        n = abs(dist) if both else max(0, -dist)
        want = n
        if n >= near:
            t = math.log(n / near) / math.log(reach / near) * (half - near)
            want = min(half - 1, near + math.floor(t + 1e-9))
        assert int(m[reach + dist]) == want + (half if both and dist > 0 else 0), dist


def test_bucket_map_refusals():
    for args in ((31, 128, True), (66, 128, True), (32, 8, True), (32, 257, True), (2, 128, True), (1, 8, False)):
        with pytest.raises(ValueError):
            sieve.relative_buckets(args[0], args[1], bidirectional=args[2], device="cpu")


def args(**kw):
    base = dict(dtype=2, heads=4, kv_heads=2, head_dim=64, nseq=3, q_tokens=100, k_tokens=100, scale=0.1, q=256, k=256,
                v=256, k_offsets=256, q_token_stride=256, q_head_stride=64, k_token_stride=128, k_head_stride=64,
                v_token_stride=128, v_head_stride=64)
    return AttentionArgsC(**{**base, **kw})


@pytest.mark.parametrize("bad", [
    dict(dtype=0), dict(dtype=3), dict(heads=3), dict(heads=0), dict(kv_heads=0), dict(head_dim=60), dict(head_dim=136),
    dict(head_dim=0), dict(nseq=-1), dict(q_tokens=-1), dict(k_tokens=99), dict(causal=2), dict(new_tokens=-1),
    dict(new_tokens=5), dict(scale=math.nan), dict(num_buckets=65, reach=8), dict(num_buckets=-1), dict(num_buckets=8, reach=257),
    dict(num_buckets=8, reach=-1), dict(nseq=0),
])
def test_attention_refuses_sizes_without_gpu(bad):
    n = C.c_size_t(77)
    for call in (sieve.lib().sieve_attention_workspace_size, sieve.lib().sieve_attention_backward_workspace_size):
        assert call(C.byref(args()), C.byref(n)) == 0 and n.value >= 256
        assert call(C.byref(args(**bad)), C.byref(n)) == -1
        assert call(None, C.byref(n)) == -1 and call(C.byref(args()), None) == -1


@pytest.mark.parametrize("bad", [
    dict(q=None), dict(q=264), dict(k=None), dict(v=8), dict(k_offsets=None), dict(q_token_stride=255), dict(v_head_stride=-64),
    dict(num_buckets=8, reach=4), dict(table=256), dict(num_buckets=8, reach=4, table=256),
])
def test_attention_refuses_pointers_without_gpu(bad):
    p = C.c_void_p(256)
    big = 1 << 40
    assert sieve.lib().sieve_attention(C.byref(args(**bad)), p, p, p, big, None) == -1
    strides = (C.c_int64 * 6)(256, 64, 128, 64, 128, 64)
    assert sieve.lib().sieve_attention_backward(C.byref(args(**bad)), p, p, p, p, p, p, strides, p, p, big, None) == -1


def test_attention_refuses_workspaces_and_outputs_without_gpu():
    lib, p, big = sieve.lib(), C.c_void_p(256), 1 << 40
    assert lib.sieve_attention(C.byref(args()), None, p, p, big, None) == -1
    assert lib.sieve_attention(C.byref(args()), p, None, p, big, None) == -1
    assert lib.sieve_attention(C.byref(args()), p, p, p, 0, None) == -3
    assert lib.sieve_attention(C.byref(args()), p, p, C.c_void_p(264), big, None) == -3
    ok = (C.c_int64 * 6)(256, 64, 128, 64, 128, 64)
    bad = (C.c_int64 * 6)(256, 60, 128, 64, 128, 64)
    assert lib.sieve_attention_backward(C.byref(args()), p, p, p, p, p, p, bad, p, p, big, None) == -1
    assert lib.sieve_attention_backward(C.byref(args()), p, p, p, p, p, p, ok, p, p, 0, None) == -3
    assert lib.sieve_attention_backward(C.byref(args(num_buckets=8, reach=4, table=256, bucket_map=256)), p, p, p, p, p, p,
                                        ok, None, p, big, None) == -1
    st = C.c_int32(5)
    assert lib.sieve_encoder_status(None, 256, C.byref(st), None) == -1
    assert lib.sieve_encoder_status(p, 128, C.byref(st), None) == -1


def test_norm_and_pool_refusals_without_gpu():
    lib, p, n = sieve.lib(), C.c_void_p(256), C.c_size_t()

    def norm(x=p, xs=64, w=p, b=p, rows=3, width=64, dtype=0, wtype=0, eps=1e-5, y=p, ys=64, m=p, r=p):
        return lib.sieve_layer_norm(x, xs, w, b, rows, width, dtype, wtype, eps, y, ys, m, r, None)
    for bad in (dict(x=None), dict(xs=63), dict(w=None), dict(rows=-1), dict(width=0), dict(width=16385), dict(dtype=3),
                dict(wtype=1), dict(eps=-1.0), dict(eps=math.inf), dict(y=None), dict(ys=10), dict(m=None),
                dict(x=C.c_void_p(258)), dict(b=C.c_void_p(258))):
        assert norm(**bad) == -1, bad
    assert lib.sieve_layer_norm_backward_workspace_size(10, 64, C.byref(n)) == 0 and n.value > 0
    assert lib.sieve_layer_norm_backward_workspace_size(-1, 64, C.byref(n)) == -1
    assert lib.sieve_layer_norm_backward(p, 64, p, 64, p, p, p, 10, 64, 0, 0, p, 64, p, p, p, 0, None) == -3
    assert lib.sieve_layer_norm_backward(p, 64, p, 64, p, None, p, 10, 64, 0, 0, p, 64, p, p, p, 1 << 30, None) == -1
    assert lib.sieve_unit_pool_workspace_size(1000, 7, 64, C.byref(n)) == 0 and n.value > 0
    for bad in ((-1, 7, 64), (1000, -1, 64), (1000, 7, 0), (1000, 7, 16385), (1 << 31, 7, 64)):
        assert lib.sieve_unit_pool_workspace_size(*bad, C.byref(n)) == -1
    assert lib.sieve_unit_pool(p, 64, None, 1000, 7, 64, 0, p, p, p, 1 << 30, None) == -1
    assert lib.sieve_unit_pool(p, 64, p, 1000, 0, 64, 0, p, p, p, 1 << 30, None) == -1
    assert lib.sieve_unit_pool(p, 64, p, 1000, 7, 64, 0, p, p, p, 0, None) == -3
    assert lib.sieve_unit_pool_backward(p, p, p, p, 1000, 7, 64, 0, p, 63, None) == -1


def test_cpu_tensors_are_refused():
    x = torch.randn(3, 8)
    for call in (lambda: sieve.layer_norm(x, torch.ones(8)), lambda: sieve.unit_pool(x, torch.tensor([0, 3], dtype=torch.int32)),
                 lambda: sieve.attention(x.half(), x.half(), x.half(), torch.tensor([0, 3], dtype=torch.int32))):
        with pytest.raises(TypeError):
            call()


def test_reference_agrees_with_autograd():
    """The reference's forward and gradients against torch's own autograd in
    64 bits, on one document with shared heads, a bias and a causal mask."""
    g = torch.Generator().manual_seed(0)
    n, heads, kv, d = 9, 4, 2, 8
    q, k, v = (torch.randn(n, h, d, generator=g).double().requires_grad_() for h in (heads, kv, kv))
    table = torch.randn(8, heads, generator=g).double().requires_grad_()
    bmap = sieve.relative_buckets(8, 6, bidirectional=False, device="cpu")
    pos = torch.arange(n)
    at = bmap.long()[(pos[None] - pos[:, None]).clamp(-6, 6) + 6]
    s = torch.einsum("ihd,jhd->hij", q, k.repeat_interleave(2, 1)) * d ** -0.5 + table[at].permute(2, 0, 1)
    s = s.masked_fill((pos[None] > pos[:, None])[None], -math.inf)
    out = torch.einsum("hij,jhd->ihd", torch.softmax(s, 2), v.repeat_interleave(2, 1))
    dout = torch.randn(n, heads, d, generator=g).double()
    want = torch.autograd.grad(out, (q, k, v, table), dout)
    ref.U[torch.float64], ref.TINY[torch.float64] = 2.0 ** -53, 1e-300
    res, _ = ref.attention(q.detach(), k.detach(), v.detach(), [n], [n], table.detach(), bmap, True, None, dout)
    for name, t in zip(("out", "dq", "dk", "dv", "dtable"), (out.detach(), *want)):
        assert torch.allclose(res[name], t, rtol=1e-10, atol=1e-12), name
    assert torch.allclose(res["lse"], torch.logsumexp(s.detach(), 2), rtol=1e-12)
    x, w, b = (torch.randn(*s_, generator=g).double().requires_grad_() for s_ in ((5, 12), (12,), (12,)))
    y = torch.nn.functional.layer_norm(x, (12,), w, b, 1e-5)
    dy = torch.randn(5, 12, generator=g).double()
    want = torch.autograd.grad(y, (x, w, b), dy)
    res, _ = ref.layer_norm(x.detach(), w.detach(), b.detach(), 1e-5, dy)
    for name, t in zip(("y", "dx", "dw", "db"), (y.detach(), *want)):
        assert torch.allclose(res[name], t, rtol=1e-9, atol=1e-11), name
    h = torch.randn(7, 6, generator=g).double().requires_grad_()
    m = torch.stack([h[:3].mean(0), h[3:].mean(0)])
    u = m / m.norm(dim=1, keepdim=True)
    dr = torch.randn(2, 6, generator=g).double()
    res, _ = ref.unit_pool(h.detach(), [3, 4], dr)
    assert torch.allclose(res["rows"], u.detach(), rtol=1e-10)
    assert torch.allclose(res["dh"], torch.autograd.grad(u, h, dr)[0], rtol=1e-9, atol=1e-12)


@pytest.mark.parametrize("reach", [-5, 7, 256, 1 << 30])
def test_reach_counts_for_nothing_without_a_table(reach):
    """Without a table the reach is not looked at: a call with a negative
    scale (which runs as if with a bias of zero) is sized and laid out the same
    whatever it holds."""
    many = dict(heads=8, kv_heads=1, nseq=4, new_tokens=1, q_tokens=4, k_tokens=1_000_000, scale=-0.5)
    sizes = []
    for r in (0, reach):
        n = C.c_size_t()
        assert sieve.lib().sieve_attention_workspace_size(C.byref(args(**many, reach=r)), C.byref(n)) == 0
        sizes.append(n.value)
    assert sizes[0] == sizes[1]


def test_unaligned_pointers_are_refused_without_gpu():
    """Every pointer that a kernel reads or writes element by element lies at
    a multiple of its element's size, or the call refuses it."""
    lib, p, odd, big = sieve.lib(), C.c_void_p(256), C.c_void_p(258), 1 << 40
    biased = dict(num_buckets=8, reach=4, table=256, bucket_map=256)
    strides = (C.c_int64 * 6)(256, 64, 128, 64, 128, 64)
    for bad in (dict(k_offsets=258), dict(q_offsets=258), dict(biased, table=258), dict(biased, bucket_map=258)):
        assert lib.sieve_attention(C.byref(args(**bad)), p, p, p, big, None) == -1, bad
        assert lib.sieve_attention_backward(C.byref(args(**bad)), p, p, p, p, p, p, strides, p, p, big, None) == -1, bad
    assert lib.sieve_attention(C.byref(args()), p, odd, p, big, None) == -1
    assert lib.sieve_attention_backward(C.byref(args()), p, p, odd, p, p, p, strides, None, p, big, None) == -1
    assert lib.sieve_attention_backward(C.byref(args(**biased)), p, p, p, p, p, p, strides, odd, p, big, None) == -1
    for m, r in ((odd, p), (p, odd)):
        assert lib.sieve_layer_norm(p, 64, p, p, 3, 64, 0, 0, 1e-5, p, 64, m, r, None) == -1
        assert lib.sieve_layer_norm_backward(p, 64, p, 64, p, m, r, 3, 64, 0, 0, p, 64, p, p, p, big, None) == -1
    for at in range(3):
        x = [odd if i == at else p for i in range(3)]
        assert lib.sieve_unit_pool(p, 64, x[0], 1000, 7, 64, 0, x[1], x[2], p, big, None) == -1, at
        assert lib.sieve_unit_pool_backward(p, x[1], x[2], x[0], 1000, 7, 64, 0, p, 64, None) == -1, at
    assert lib.sieve_unit_pool_backward(odd, p, p, p, 1000, 7, 64, 0, p, 64, None) == -1


@pytest.mark.parametrize("name", ["q_token_stride", "q_head_stride", "k_token_stride", "k_head_stride", "v_token_stride",
                                  "v_head_stride"])
@pytest.mark.parametrize("stride", [0, 56])
def test_overlapping_heads_are_refused_without_gpu(name, stride):
    """A stride of zero (an expanded tensor) or below the head's length, where
    the axis has more than one element; where it has one, any."""
    p, big, fields = C.c_void_p(256), 1 << 40, ["q_token_stride", "q_head_stride", "k_token_stride", "k_head_stride",
                                                "v_token_stride", "v_head_stride"]
    lib = sieve.lib()
    assert lib.sieve_attention(C.byref(args(**{name: stride})), p, p, p, big, None) == -1
    strides = [256, 64, 128, 64, 128, 64]
    strides[fields.index(name)] = stride
    assert lib.sieve_attention_backward(C.byref(args()), p, p, p, p, p, p, (C.c_int64 * 6)(*strides), p, p, big, None) == -1
    single = args(**{name: stride}, heads=1, kv_heads=1, nseq=1, q_tokens=1, k_tokens=1)
    assert lib.sieve_attention(C.byref(single), p, p, p, 0, None) == -3          # only the workspace is wrong


def test_binding_names_expanded_tensors():
    t = torch.empty(5, 1, 64).expand(5, 3, 64)
    for call in (lambda: sieve.encoder._strides(t), lambda: sieve.encoder._new_strides(torch.empty(1, 1, 3, 64).expand(4, 1, 3, 64))):
        with pytest.raises(ValueError, match="contiguous"):
            call()
    assert sieve.encoder._strides(torch.empty(1, 3, 64)[:, :1]) == (64, 64)
