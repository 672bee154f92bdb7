"""Encoder operators: what turns packed documents into the unit rows that the
search takes, and the backward passes that train it (C ABI:
``include/sieve_encoder.h``).

Documents are packed one after the other without padding; ``offsets`` (int32,
device, ``[nseq + 1]``) holds where each starts and where the last ends.  As
everywhere in this package the functions only marshal tensors into libsieve's
CUDA kernels; they raise TypeError or ValueError for tensors they cannot take
and :class:`SieveError` for anything the library refuses, and run on
``stream`` (default: the current stream of the tensors' device).  Results and
scratch belong to the stream they are computed on; with an explicit ``stream``
inputs are kept from reuse until that stream has passed the call.  Rows that
belong to no document (before the first offset, past the last) are not written
in results: a tensor with room to spare holds anything there.

The calls are outside of torch.autograd: results never require a gradient,
whatever their inputs do, and a backward pass is a call of its own, as in
``examples/encode_and_deduplicate.py``.

* :func:`layer_norm`, :func:`layer_norm_backward`
* :func:`attention`, :func:`attention_backward` (relative position bias:
  :func:`relative_buckets`)
* :func:`unit_pool`, :func:`unit_pool_backward`
"""
from __future__ import annotations

import contextlib
import ctypes as C

import torch

import paper_2608_03199_gb300 as _sieve

DTYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
MAX_BUCKETS = 64
MAX_REACH = 256


class AttentionArgsC(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("heads", C.c_int32), ("kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("nseq", C.c_int64), ("q_tokens", C.c_int64), ("k_tokens", C.c_int64),
                ("new_tokens", C.c_int32), ("causal", C.c_int32), ("scale", C.c_float),
                ("num_buckets", C.c_int32), ("reach", C.c_int32), ("reserved0", C.c_int32),
                ("q_offsets", C.c_void_p), ("k_offsets", C.c_void_p),
                ("q", C.c_void_p), ("k", C.c_void_p), ("v", C.c_void_p),
                ("q_token_stride", C.c_int64), ("q_head_stride", C.c_int64),
                ("k_token_stride", C.c_int64), ("k_head_stride", C.c_int64),
                ("v_token_stride", C.c_int64), ("v_head_stride", C.c_int64),
                ("table", C.c_void_p), ("bucket_map", C.c_void_p)]


_p, _i32, _i64, _size = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
SIGNATURES = {
    "sieve_layer_norm": (_i32, [_p, _i64, _p, _p, _i64, _i32, _i32, _i32, C.c_float, _p, _i64, _p, _p, _p]),
    "sieve_layer_norm_backward_workspace_size": (_i32, [_i64, _i32, C.POINTER(_size)]),
    "sieve_layer_norm_backward": (_i32, [_p, _i64, _p, _i64, _p, _p, _p, _i64, _i32, _i32, _i32, _p, _i64, _p,
                                         _p, _p, _size, _p]),
    "sieve_attention_workspace_size": (_i32, [C.POINTER(AttentionArgsC), C.POINTER(_size)]),
    "sieve_attention": (_i32, [C.POINTER(AttentionArgsC), _p, _p, _p, _size, _p]),
    "sieve_attention_backward_workspace_size": (_i32, [C.POINTER(AttentionArgsC), C.POINTER(_size)]),
    "sieve_attention_backward": (_i32, [C.POINTER(AttentionArgsC), _p, _p, _p, _p, _p, _p, _p, _p, _p, _size, _p]),
    "sieve_encoder_status": (_i32, [_p, _size, C.POINTER(_i32), _p]),
    "sieve_unit_pool_workspace_size": (_i32, [_i64, _i64, _i32, C.POINTER(_size)]),
    "sieve_unit_pool": (_i32, [_p, _i64, _p, _i64, _i64, _i32, _i32, _p, _p, _p, _size, _p]),
    "sieve_unit_pool_backward": (_i32, [_p, _p, _p, _p, _i64, _i64, _i32, _i32, _p, _i64, _p]),
}


@contextlib.contextmanager
def _on(device, stream, inputs):
    """Allocations inside belong to ``stream``; ``inputs`` allocated on
    another stream are kept until ``stream`` has passed the call."""
    with torch.cuda.device(device), torch.cuda.stream(stream):
        yield stream.cuda_stream
        for t in inputs:
            if t is not None:
                t.record_stream(stream)


@contextlib.contextmanager
def _on_device(device):
    with torch.cuda.device(device):
        yield torch.cuda.current_stream(device).cuda_stream


class _Current:
    """The usual case, without a context switch: the current stream of the
    current device."""
    __slots__ = ("handle",)

    def __init__(self, handle):
        self.handle = handle

    def __enter__(self):
        return self.handle

    def __exit__(self, *exc):
        return False


def _launch(device, stream, *inputs):
    if stream is not None:
        return _on(device, stream, inputs)
    index = device.index
    if index != torch._C._cuda_getDevice():
        return _on_device(device)
    return _Current(torch._C._cuda_getCurrentRawStream(index))


def _need(t, name, dtypes, ndim, device=None):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    if t.dtype not in dtypes:
        raise TypeError(f"{name} must be {' or '.join(str(d) for d in dtypes)}, got {t.dtype}")
    if ndim is not None and t.dim() != ndim:
        raise ValueError(f"{name} must have {ndim} dims, has {t.dim()}")
    if device is not None and t.device != device:
        raise ValueError(f"{name} is on {t.device}, expected {device}")
    return t


def _rows(t, name, dtypes, device=None, shape=None):
    """(rows, width, row stride) of a matrix whose rows are contiguous (their
    stride is free); a contiguous tensor of more dims counts as the matrix of
    its last axis."""
    _need(t, name, dtypes, None, device)
    size = t.shape
    if shape is not None and size != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, has {tuple(size)}")
    if len(size) < 1:
        raise ValueError(f"{name} must be contiguous or a matrix")
    width = size[-1]
    if t.is_contiguous():
        rows = size[0] if len(size) == 2 else t.numel() // width if width else 0
        return rows, width, width
    if len(size) != 2:
        raise ValueError(f"{name} must be contiguous or a matrix")
    rows, (across, along) = size[0], t.stride()
    if width > 1 and along != 1:
        raise ValueError(f"{name}: the elements of a row must be contiguous")
    if rows > 1 and across < width:
        raise ValueError(f"{name}: rows must not overlap")
    return rows, width, across if rows > 1 else width


def _vector(t, name, dtypes, n, device):
    _need(t, name, dtypes, 1, device)
    if t.shape[0] != n or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous with {n} elements")
    return t


def _offsets(t, name, device, n=None):
    _need(t, name, (torch.int32,), 1, device)
    if t.shape[0] < 1 or not t.is_contiguous() or (n is not None and t.shape[0] != n):
        raise ValueError(f"{name} must be a contiguous [nseq + 1] tensor")
    return t


def _scratch(workspace, nbytes, device):
    if workspace is not None:
        return workspace.get(nbytes, device)
    return torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)


_FLOATS = tuple(DTYPES)
_HALVES = (torch.float16, torch.bfloat16)


# ---------------------------------------------------------------------------
def layer_norm(x, weight, bias=None, eps=1e-5, out=None, stream=None):
    """Layer norm over the last axis of ``x`` (fp32, fp16 or bf16):
    y = (x - mean) rstd weight + bias (sieve_layer_norm).

    ``x``: a matrix with contiguous rows of any stride, or a contiguous tensor
    of more dims.  ``weight`` / ``bias``: [width] of x's type or fp32.
    Returns (y, mean, rstd); mean and rstd ([rows] fp32) are what
    :func:`layer_norm_backward` needs."""
    rows, width, xs = _rows(x, "x", _FLOATS)
    dev, kind = x.device, x.dtype
    _vector(weight, "weight", (kind, torch.float32), width, dev)
    if bias is not None:
        _vector(bias, "bias", (weight.dtype,), width, dev)
    with _launch(dev, stream, x, weight, bias, out) as s:
        if out is None:
            out, ys = torch.empty(x.shape, dtype=kind, device=dev), width
        else:
            ys = _rows(out, "out", (kind,), dev, x.shape)[2]
        mean = torch.empty(rows, dtype=torch.float32, device=dev)
        rstd = torch.empty(rows, dtype=torch.float32, device=dev)
        rc = _sieve.lib().sieve_layer_norm(
            x.data_ptr(), xs, weight.data_ptr(), None if bias is None else bias.data_ptr(), rows, width,
            DTYPES[kind], DTYPES[weight.dtype], eps, out.data_ptr(), ys, mean.data_ptr(), rstd.data_ptr(), s)
        if rc:
            _sieve._check(rc, "sieve_layer_norm")
    return out, mean, rstd


def layer_norm_backward(dy, x, weight, mean, rstd, need_dbias=True, out=None, workspace=None, stream=None):
    """Gradients of :func:`layer_norm`: (dx, dweight, dbias), dbias None
    without ``need_dbias`` (sieve_layer_norm_backward).  ``mean`` and ``rstd``
    are the forward call's; ``out`` receives dx and may be ``dy``."""
    rows, width, xs = _rows(x, "x", _FLOATS)
    dev = x.device
    dys = _rows(dy, "dy", (x.dtype,), dev, x.shape)[2]
    _vector(weight, "weight", (x.dtype, torch.float32), width, dev)
    _vector(mean, "mean", (torch.float32,), rows, dev)
    _vector(rstd, "rstd", (torch.float32,), rows, dev)
    lib = _sieve.lib()
    n = _size()
    _sieve._check(lib.sieve_layer_norm_backward_workspace_size(rows, width, C.byref(n)),
                  "sieve_layer_norm_backward_workspace_size")
    with _launch(dev, stream, dy, x, weight, mean, rstd, out) as s:
        if out is None:
            out = torch.empty(x.shape, dtype=x.dtype, device=dev)
        dxs = _rows(out, "out", (x.dtype,), dev, x.shape)[2]
        dw = torch.empty(width, dtype=weight.dtype, device=dev)
        db = torch.empty(width, dtype=weight.dtype, device=dev) if need_dbias else None
        ws = _scratch(workspace, n.value, dev)
        _sieve._check(lib.sieve_layer_norm_backward(
            dy.data_ptr(), dys, x.data_ptr(), xs, weight.data_ptr(), mean.data_ptr(), rstd.data_ptr(), rows,
            width, DTYPES[x.dtype], DTYPES[weight.dtype], out.data_ptr(), dxs, dw.data_ptr(),
            None if db is None else db.data_ptr(), ws.data_ptr(), ws.numel(), s), "sieve_layer_norm_backward")
    return out, dw, db


# ---------------------------------------------------------------------------
def relative_buckets(num_buckets, max_distance, bidirectional=True, device=None):
    """The bucket of every distance key - query in [-max_distance,
    max_distance], as the int32 map :func:`attention` takes.

    Half of the buckets hold one near distance each, the rest distances up to
    max_distance on a logarithmic scale: distance n >= e (e the number of near
    ones) is in bucket e + floor(far * log(n / e) / log(max_distance / e)),
    the last one also holding everything farther.  ``bidirectional`` gives
    each direction half of the buckets (the second half to keys after the
    query); otherwise keys after the query share bucket 0.  The bounds are
    found in whole numbers, so no distance depends on a rounding."""
    half = num_buckets // 2 if bidirectional else num_buckets
    if (bidirectional and num_buckets % 2) or half < 2 or num_buckets > MAX_BUCKETS:
        raise ValueError(f"num_buckets must be at least {4 if bidirectional else 2}, even for both directions, and "
                         f"at most {MAX_BUCKETS}, got {num_buckets}")
    near = half // 2
    far = half - near
    if not near < max_distance <= MAX_REACH:
        raise ValueError(f"max_distance must be above {near} and at most {MAX_REACH}, got {max_distance}")

    def bucket(n):
        if n < near:
            return n
        t = 0
        while t + 1 < far and n ** far * near ** (t + 1) >= max_distance ** (t + 1) * near ** far:
            t += 1
        return near + t

    side = [bucket(n) for n in range(max_distance + 1)]
    behind = side[:0:-1] + [side[0]]
    ahead = [half + b for b in side[1:]] if bidirectional else [0] * max_distance
    return torch.tensor(behind + ahead, dtype=torch.int32).to("cuda" if device is None else device)


def _heads(t, name, dtypes, device, ndim=3):
    _need(t, name, dtypes, ndim, device)
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError(f"{name}: the elements of a head must be contiguous")
    return t


def _strides(t):
    """Token and head strides; an axis of one element has none that matters."""
    *_, tokens, heads, dim = t.shape
    *_, ts, hs, _ = t.stride()
    return _apart(ts if tokens > 1 else heads * dim, hs if heads > 1 else dim, dim)


def _apart(ts, hs, dim):
    if ts < dim or hs < dim:
        raise ValueError("tokens and heads must not overlap: an expanded tensor has to be made contiguous")
    return ts, hs


def _new_strides(t):
    """The same of [nseq][new][heads][dim], whose tokens must be evenly spaced."""
    nseq, new, heads, dim = t.shape
    across, ts, hs, _ = t.stride()
    if nseq > 1 and new > 1 and across != new * ts:
        raise ValueError("new tokens must be evenly spaced")
    return _apart(across if new == 1 and nseq > 1 else ts if new > 1 else heads * dim, hs if heads > 1 else dim, dim)


def _attention_args(q, k, v, offsets, q_offsets, table, buckets, causal, scale):
    _need(q, "q", _HALVES, None)
    dev, kind = q.device, (q.dtype,)
    ndim = q.dim()
    if ndim != 3 and ndim != 4:
        raise ValueError("q must be [tokens][heads][dim] or [nseq][new][heads][dim]")
    _heads(q, "q", kind, None, ndim)
    _heads(k, "k", kind, dev)
    _heads(v, "v", kind, dev)
    _offsets(offsets, "offsets", dev)
    nseq = offsets.shape[0] - 1
    heads, dim = q.shape[-2:]
    k_tokens, kv_heads, k_dim = k.shape
    if v.shape != k.shape or k_dim != dim or heads % max(kv_heads, 1):
        raise ValueError(f"q {tuple(q.shape)}, k {tuple(k.shape)} and v {tuple(v.shape)} do not fit together")
    new, q_off = 0, None
    if ndim == 4:
        if q_offsets is not None:
            raise ValueError("q of [nseq][new][heads][dim] has no q_offsets")
        new = q.shape[1]
        if q.shape[0] != nseq or new < 1:
            raise ValueError("q must hold the same number of new tokens, at least one, for every document")
        q_tokens = nseq * new
        q_ts, q_hs = _new_strides(q)
    else:
        q_tokens = q.shape[0]
        q_ts, q_hs = _strides(q)
        if q_offsets is not None:
            q_off = _offsets(q_offsets, "q_offsets", dev, nseq + 1).data_ptr()
        elif q_tokens != k_tokens:
            raise ValueError("q and k hold different numbers of tokens: pass q_offsets")
    if (table is None) != (buckets is None):
        raise ValueError("table and buckets go together")
    bias = (0, 0, None, None)
    if table is not None:
        _need(table, "table", (torch.float32,), 2, dev)
        _need(buckets, "buckets", (torch.int32,), 1, dev)
        if table.shape[1] != heads or not table.is_contiguous():
            raise ValueError(f"table must be contiguous [num_buckets][{heads}]")
        if buckets.shape[0] % 2 != 1 or not buckets.is_contiguous():
            raise ValueError("buckets must be contiguous [2 reach + 1]")
        if table.shape[0] < 1:
            raise ValueError("table has no bucket")
        bias = (table.shape[0], buckets.shape[0] // 2, table.data_ptr(), buckets.data_ptr())
    return AttentionArgsC(DTYPES[q.dtype], heads, kv_heads, dim, nseq, q_tokens, k_tokens, new, 1 if causal else 0,
                          dim ** -0.5 if scale is None and dim else scale or 0.0, bias[0], bias[1], 0, q_off,
                          offsets.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(), q_ts, q_hs, *_strides(k),
                          *_strides(v), bias[2], bias[3])


def attention(q, k, v, offsets, q_offsets=None, table=None, buckets=None, causal=False, scale=None, out=None,
              workspace=None, stream=None, check=False):
    """Attention over packed documents (sieve_attention), fp16 or bf16.

    ``q`` [tokens][heads][dim], ``k`` and ``v`` [tokens][kv_heads][dim] (heads
    a multiple of kv_heads; dim a multiple of 8 up to 128), token and head
    strides free, so parts of one projection work.  ``offsets``: the documents
    of k and v; q has the same unless ``q_offsets`` says otherwise.  For the
    next tokens of growing documents pass ``q`` as [nseq][new][heads][dim].
    The last query of a document stands at its last key.

    ``table`` [num_buckets][heads] fp32 with ``buckets``
    (:func:`relative_buckets`): the learned bias of each bucket of distances.
    ``causal``: a query sees the keys up to its own place.  ``scale`` defaults
    to dim ** -0.5.  ``check``: read the device status afterwards
    (synchronizes) and raise if a bounded wait gave up.

    Returns (out like q, lse [heads][query tokens] fp32); a query that sees no
    key gets zeros and -inf."""
    a = _attention_args(q, k, v, offsets, q_offsets, table, buckets, causal, scale)
    dev = q.device
    lib = _sieve.lib()
    n = _size()
    ref = C.byref(a)
    rc = lib.sieve_attention_workspace_size(ref, C.byref(n))
    if rc:
        _sieve._check(rc, "sieve_attention_workspace_size")
    with _launch(dev, stream, q, k, v, offsets, q_offsets, table, buckets, out) as s:
        if out is None:
            out = torch.empty(q.shape, dtype=q.dtype, device=dev)
        elif out.shape != q.shape or out.dtype != q.dtype or out.device != dev or not out.is_contiguous():
            raise ValueError("out must be contiguous, of q's shape and type")
        lse = torch.empty((a.heads, a.q_tokens), dtype=torch.float32, device=dev)
        ws = _scratch(workspace, n.value, dev)
        rc = lib.sieve_attention(ref, out.data_ptr(), lse.data_ptr(), ws.data_ptr(), ws.numel(), s)
        if rc:
            _sieve._check(rc, "sieve_attention")
        if check and a.q_tokens:
            _sieve._check(encoder_status(ws, s), "sieve_attention (device status)")
    return out, lse


def attention_backward(dout, q, k, v, out, lse, offsets, q_offsets=None, table=None, buckets=None, causal=False,
                       scale=None, grads=None, workspace=None, stream=None, check=False):
    """Gradients of :func:`attention`: (dq, dk, dv, dtable), dtable fp32, None
    without a table (sieve_attention_backward).

    ``out`` and ``lse`` are the forward call's, the other arguments the same
    as there.  ``grads``: (dq, dk, dv) to write into, with free token and head
    strides, e.g. parts of one projection's gradient."""
    a = _attention_args(q, k, v, offsets, q_offsets, table, buckets, causal, scale)
    dev = q.device
    for t, name in ((dout, "dout"), (out, "out")):
        _need(t, name, (q.dtype,), q.dim(), dev)
        if t.shape != q.shape:
            raise ValueError(f"{name} must have q's shape")
    if not out.is_contiguous():
        raise ValueError("out must be contiguous")
    _need(lse, "lse", (torch.float32,), 2, dev)
    if tuple(lse.shape) != (a.heads, a.q_tokens) or not lse.is_contiguous():
        raise ValueError("lse must be the forward call's")
    lib = _sieve.lib()
    n = _size()
    _sieve._check(lib.sieve_attention_backward_workspace_size(C.byref(a), C.byref(n)),
                  "sieve_attention_backward_workspace_size")
    with _launch(dev, stream, dout, q, k, v, out, lse, offsets, q_offsets, table, buckets, *(grads or ())) as s:
        dout = dout.contiguous()
        if grads is None:
            grads = tuple(torch.empty(t.shape, dtype=t.dtype, device=dev) for t in (q, k, v))
        strides = []
        for g, t, name in zip(grads, (q, k, v), ("dq", "dk", "dv")):
            _heads(g, name, (q.dtype,), dev, t.dim())
            if g.shape != t.shape:
                raise ValueError(f"{name} must have shape {tuple(t.shape)}")
            strides += _new_strides(g) if g.dim() == 4 else _strides(g)
        dtable = None if table is None else torch.empty(table.shape, dtype=torch.float32, device=dev)
        ws = _scratch(workspace, n.value, dev)
        _sieve._check(lib.sieve_attention_backward(
            C.byref(a), dout.data_ptr(), out.data_ptr(), lse.data_ptr(), grads[0].data_ptr(), grads[1].data_ptr(),
            grads[2].data_ptr(), (_i64 * 6)(*strides), None if dtable is None else dtable.data_ptr(),
            ws.data_ptr(), ws.numel(), s), "sieve_attention_backward")
        if check and (a.q_tokens or a.k_tokens):
            _sieve._check(encoder_status(ws, s), "sieve_attention_backward (device status)")
    return grads[0], grads[1], grads[2], dtable


def encoder_status(ws, stream) -> int:
    """The device status word of the last attention call that used the
    workspace tensor ``ws`` (sieve_encoder_status; synchronizes the stream)."""
    v = _i32(0)
    handle = stream if isinstance(stream, int) else _sieve._stream(stream)
    buf = ws.buf if isinstance(ws, _sieve.Workspace) else ws
    _sieve._check(_sieve.lib().sieve_encoder_status(buf.data_ptr(), buf.numel(), C.byref(v), handle),
                  "sieve_encoder_status")
    return int(v.value)


# ---------------------------------------------------------------------------
def unit_pool(h, offsets, out=None, workspace=None, stream=None):
    """One unit-norm fp32 row per document, the direction of the mean of its
    tokens' rows in ``h`` [tokens][width] (fp32, fp16 or bf16): what
    :func:`search` takes (sieve_unit_pool).  Returns (rows [nseq][width],
    norms [nseq], the means' lengths); a document without tokens, or whose
    mean is zero, gets zeros."""
    tokens, width, hs = _rows(h, "h", _FLOATS)
    if h.dim() != 2:
        raise ValueError("h must be [tokens][width]")
    dev = h.device
    _offsets(offsets, "offsets", dev)
    nseq = offsets.shape[0] - 1
    lib = _sieve.lib()
    n = _size()
    _sieve._check(lib.sieve_unit_pool_workspace_size(tokens, nseq, width, C.byref(n)),
                  "sieve_unit_pool_workspace_size")
    with _launch(dev, stream, h, offsets, out) as s:
        if out is None:
            out = torch.empty((nseq, width), dtype=torch.float32, device=dev)
        elif tuple(out.shape) != (nseq, width) or out.dtype != torch.float32 or out.device != dev \
                or not out.is_contiguous():
            raise ValueError("out must be a contiguous float32 [nseq][width] tensor")
        norms = torch.empty(nseq, dtype=torch.float32, device=dev)
        ws = _scratch(workspace, n.value, dev)
        _sieve._check(lib.sieve_unit_pool(h.data_ptr(), hs, offsets.data_ptr(), tokens, nseq, width,
                                          DTYPES[h.dtype], out.data_ptr(), norms.data_ptr(), ws.data_ptr(),
                                          ws.numel(), s), "sieve_unit_pool")
    return out, norms


def unit_pool_backward(drows, rows, norms, offsets, tokens, dtype=torch.float32, out=None, stream=None):
    """Gradient of :func:`unit_pool` for its input: dh [tokens][width] of
    ``dtype`` (sieve_unit_pool_backward).  ``rows`` and ``norms`` are the
    forward call's results, ``tokens`` the number of its input's rows."""
    dev = rows.device
    _need(rows, "rows", (torch.float32,), 2)
    nseq, width = rows.shape
    _need(drows, "drows", (torch.float32,), 2, dev)
    if drows.shape != rows.shape or not rows.is_contiguous():
        raise ValueError("drows and rows must have the same shape, rows contiguous")
    _vector(norms, "norms", (torch.float32,), nseq, dev)
    _offsets(offsets, "offsets", dev, nseq + 1)
    if dtype not in DTYPES:
        raise TypeError(f"dtype must be one of {', '.join(str(d) for d in DTYPES)}")
    with _launch(dev, stream, drows, rows, norms, offsets, out) as s:
        drows = drows.contiguous()
        if out is None:
            out = torch.empty((tokens, width), dtype=dtype, device=dev)
        hs = _rows(out, "out", (dtype,), dev, torch.Size((tokens, width)))[2]
        _sieve._check(_sieve.lib().sieve_unit_pool_backward(
            drows.data_ptr(), rows.data_ptr(), norms.data_ptr(), offsets.data_ptr(), tokens, nseq, width,
            DTYPES[dtype], out.data_ptr(), hs, s), "sieve_unit_pool_backward")
    return out
