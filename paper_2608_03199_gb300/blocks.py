"""The operators around an encoder's blocks: from token ids to the first
hidden states, from one block to the next, and from the last hidden states to
the loss, with their backward passes (C ABI: ``include/sieve_encoder.h``).

The conventions are :mod:`paper_2608_03199_gb300.encoder`'s: the functions only
marshal tensors into libsieve's CUDA kernels, raise TypeError or ValueError for
tensors they cannot take and :class:`SieveError` for anything the library
refuses, run on ``stream`` (default: the current stream of the tensors'
device), and are outside of torch.autograd.

* :func:`embed`, :func:`embed_backward`
* :func:`residual_norm`, :func:`residual_norm_backward`
* :func:`cross_entropy`, :func:`cross_entropy_backward`
"""
from __future__ import annotations

import ctypes as C

import torch

import paper_2608_03199_gb300 as _sieve
from .encoder import (DTYPES, _FLOATS, _HALVES, _launch, _need, _rows, _scratch, _vector, encoder_status)

ID_TYPES = {torch.int32: 3, torch.int64: 4}


class ResidualNormArgsC(C.Structure):
    _fields_ = [("rows", C.c_int64), ("width", C.c_int32), ("dtype", C.c_int32), ("weight_dtype", C.c_int32),
                ("rms", C.c_int32), ("gate_kind", C.c_int32), ("alpha", C.c_float), ("eps", C.c_float),
                ("reserved0", C.c_int32),
                ("h", C.c_void_p), ("y", C.c_void_p), ("gate", C.c_void_p),
                ("h_stride", C.c_int64), ("y_stride", C.c_int64), ("gate_stride", C.c_int64),
                ("weight", C.c_void_p), ("bias", C.c_void_p), ("post_weight", C.c_void_p), ("post_bias", C.c_void_p)]


class ResidualNormGradsC(C.Structure):
    _fields_ = [("dstream", C.c_void_p), ("dx", C.c_void_p), ("dstream_stride", C.c_int64), ("dx_stride", C.c_int64),
                ("stats", C.c_void_p), ("dh", C.c_void_p), ("dy", C.c_void_p), ("dgate", C.c_void_p),
                ("dh_stride", C.c_int64), ("dy_stride", C.c_int64), ("dgate_stride", C.c_int64),
                ("dweight", C.c_void_p), ("dbias", C.c_void_p), ("dpost_weight", C.c_void_p),
                ("dpost_bias", C.c_void_p)]


class CrossEntropyArgsC(C.Structure):
    _fields_ = [("rows", C.c_int64), ("classes", C.c_int64), ("width", C.c_int32), ("dtype", C.c_int32),
                ("target_type", C.c_int32), ("scale", C.c_float),
                ("h", C.c_void_p), ("weight", C.c_void_p), ("h_stride", C.c_int64), ("weight_stride", C.c_int64),
                ("bias", C.c_void_p), ("targets", C.c_void_p), ("wait_limit", C.c_int32), ("reserved0", C.c_int32)]


class CrossEntropyGradsC(C.Structure):
    _fields_ = [("dloss", C.c_void_p), ("loss", C.c_void_p), ("lse", C.c_void_p), ("dh", C.c_void_p),
                ("dweight", C.c_void_p), ("dh_stride", C.c_int64), ("dweight_stride", C.c_int64),
                ("dweight_dtype", C.c_int32), ("accumulate", C.c_int32), ("dbias", C.c_void_p)]


_p, _i32, _i64, _size, _f = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t, C.c_float
_norm_ref, _loss_ref = C.POINTER(ResidualNormArgsC), C.POINTER(CrossEntropyArgsC)
SIGNATURES = {
    "sieve_embed": (_i32, [_p, _i32, _i64, _p, _i64, _i64, _i32, _i32, _f, _p, _i64, _i32, _p]),
    "sieve_embed_backward_workspace_size": (_i32, [_i64, _i64, _i32, C.POINTER(_size)]),
    "sieve_embed_backward": (_i32, [_p, _i64, _p, _i32, _i64, _i64, _i32, _i32, _f, _p, _i64, _i32, _i32, _p, _size,
                                    _p]),
    "sieve_residual_norm": (_i32, [_norm_ref, _p, _i64, _p, _i64, _p, _p]),
    "sieve_residual_norm_backward_workspace_size": (_i32, [_i64, _i32, C.POINTER(_size)]),
    "sieve_residual_norm_backward": (_i32, [_norm_ref, C.POINTER(ResidualNormGradsC), _p, _size, _p]),
    "sieve_cross_entropy_workspace_size": (_i32, [_loss_ref, C.POINTER(_size)]),
    "sieve_cross_entropy": (_i32, [_loss_ref, _p, _p, _p, _size, _p]),
    "sieve_cross_entropy_backward_workspace_size": (_i32, [_loss_ref, C.POINTER(_size)]),
    "sieve_cross_entropy_backward": (_i32, [_loss_ref, C.POINTER(CrossEntropyGradsC), _p, _size, _p]),
}


def _ptr(t):
    return None if t is None else t.data_ptr()


def _ids(t, name, device=None, n=None):
    _need(t, name, tuple(ID_TYPES), None, device)
    if not t.is_contiguous() or (n is not None and (t.dim() != 1 or t.shape[0] != n)):
        raise ValueError(f"{name} must be contiguous" + ("" if n is None else f" with {n} elements"))
    return t


def _tiles(t, name, dtypes, device=None, shape=None):
    """(rows, width, row stride) of a matrix that bulk copies take: rows at
    multiples of 16 bytes."""
    _need(t, name, dtypes, 2, device)
    got = _rows(t, name, dtypes, device, shape)
    per = 16 // t.element_size()
    if got[0] and (t.data_ptr() % 16 or (got[0] > 1 and got[2] % max(per, 8))):
        raise ValueError(f"{name}: rows must start at multiples of 16 bytes and lie a multiple of 8 elements apart")
    return got


# ---------------------------------------------------------------------------
def embed(ids, table, scale=1.0, dtype=None, out=None, stream=None):
    """The rows of ``table`` [vocab][width] (fp32, fp16 or bf16, row stride
    free) that ``ids`` (int32 or int64, contiguous, any shape) name, times
    ``scale``, as [*ids.shape][width] of ``dtype`` (default: the table's)
    (sieve_embed).  An id outside [0, vocab) gives zeros."""
    _need(table, "table", _FLOATS, 2)
    vocab, width, ts = _rows(table, "table", _FLOATS)
    dev = table.device
    _ids(ids, "ids", dev)
    dtype = table.dtype if dtype is None else dtype
    if dtype not in DTYPES:
        raise TypeError(f"dtype must be one of {', '.join(str(d) for d in DTYPES)}")
    shape = torch.Size((*ids.shape, width))
    with _launch(dev, stream, ids, table, out) as s:
        if out is None:
            out = torch.empty(shape, dtype=dtype, device=dev)
        os = _rows(out, "out", (dtype,), dev, shape)[2]
        rc = _sieve.lib().sieve_embed(ids.data_ptr(), ID_TYPES[ids.dtype], ids.numel(), table.data_ptr(), ts, vocab,
                                      width, DTYPES[table.dtype], scale, out.data_ptr(), os, DTYPES[dtype], s)
        if rc:
            _sieve._check(rc, "sieve_embed")
    return out


def embed_backward(dout, ids, vocab, scale=1.0, dtype=torch.float32, out=None, accumulate=False, workspace=None,
                   stream=None):
    """The gradient of :func:`embed` for its table, [vocab][width] of
    ``dtype`` (sieve_embed_backward): row v is ``scale`` times the sum of
    ``dout`` over the tokens whose id is v, added up in fp32: the tokens sorted
    by id are cut into pieces of 64, each of which adds its tokens up in order; an
    id's pieces are then added up in an order that depends on the ids alone.
    ``accumulate``: add to ``out``, where rows without a token stay as
    they are; else they are zeros."""
    tokens, width, ds = _rows(dout, "dout", _FLOATS)
    dev = dout.device
    _ids(ids, "ids", dev)
    if dout.dim() < 2 or dout.shape[:-1] != (ids.shape if dout.dim() > 2 else (ids.numel(),)):
        raise ValueError(f"dout {tuple(dout.shape)} and ids {tuple(ids.shape)} do not fit together")
    if dtype not in DTYPES:
        raise TypeError(f"dtype must be one of {', '.join(str(d) for d in DTYPES)}")
    if accumulate and out is None:
        raise ValueError("accumulate adds to out, which is missing")
    tokens = ids.numel()
    lib = _sieve.lib()
    n = _size()
    _sieve._check(lib.sieve_embed_backward_workspace_size(tokens, vocab, width, C.byref(n)),
                  "sieve_embed_backward_workspace_size")
    with _launch(dev, stream, dout, ids, out) as s:
        if out is None:
            out = torch.empty((vocab, width), dtype=dtype, device=dev)
        elif out.dtype in DTYPES:
            dtype = out.dtype
        gs = _rows(out, "out", (dtype,), dev, torch.Size((vocab, width)))[2]
        ws = _scratch(workspace, n.value, dev)
        _sieve._check(lib.sieve_embed_backward(
            dout.data_ptr(), ds, ids.data_ptr(), ID_TYPES[ids.dtype], tokens, vocab, width, DTYPES[dout.dtype], scale,
            out.data_ptr(), gs, DTYPES[dtype], 1 if accumulate else 0, ws.data_ptr(), ws.numel(), s),
            "sieve_embed_backward")
    return out


# ---------------------------------------------------------------------------
def _residual_args(h, y, weight, bias, post_weight, post_bias, gate, alpha, rms, eps):
    rows, width, hs = _rows(h, "h", _FLOATS)
    dev, kind = h.device, h.dtype
    ys = _rows(y, "y", (kind,), dev, h.shape)[2]
    if weight is None and post_weight is None:
        raise ValueError("at least one of weight and post_weight is needed")
    first = weight if weight is not None else post_weight
    wtype = first.dtype if isinstance(first, torch.Tensor) else None
    if wtype is not kind and wtype is not torch.float32:
        _need(first, "weight" if weight is not None else "post_weight", (kind, torch.float32), 1, dev)
    types = (wtype,)
    if weight is not None:
        _vector(weight, "weight", types, width, dev)
    if bias is not None:
        if weight is None:
            raise ValueError("a bias goes with its weight: weight is missing")
        _vector(bias, "bias", types, width, dev)
    if post_weight is not None:
        _vector(post_weight, "post_weight", types, width, dev)
    if post_bias is not None:
        if post_weight is None:
            raise ValueError("a bias goes with its weight: post_weight is missing")
        _vector(post_bias, "post_bias", types, width, dev)
    gate_kind, gs = 0, 0
    if gate is not None:
        if isinstance(gate, torch.Tensor) and gate.dim() == 1 and h.dim() > 1:
            gate_kind = 1
            _vector(gate, "gate", types, width, dev)
        else:
            gate_kind = 2
            gs = _rows(gate, "gate", (kind,), dev, h.shape)[2]
    return ResidualNormArgsC(rows, width, DTYPES[kind], DTYPES[wtype], 1 if rms else 0, gate_kind, alpha, eps, 0,
                             h.data_ptr(), y.data_ptr(), _ptr(gate), hs, ys, gs, _ptr(weight), _ptr(bias),
                             _ptr(post_weight), _ptr(post_bias))


def residual_norm(h, y, weight=None, bias=None, post_weight=None, post_bias=None, gate=None, alpha=1.0, eps=1e-5,
                  rms=False, out=None, x_out=None, stream=None):
    """The residual step between two blocks (sieve_residual_norm): a block's
    output ``y`` is normed with ``post_weight`` and ``post_bias`` (if given),
    multiplied by ``gate`` (if given: [width], or one for every element of
    h's shape and type) and added to ``alpha`` times the stream ``h``; the sum
    is the new stream, and normed with ``weight`` and ``bias`` (if given) the
    next block's input x.

    h and y: matrices with contiguous rows of any stride, or contiguous tensors
    of more dims, fp32, fp16 or bf16; the weights, biases and a gate of [width]
    of one type, h's or fp32.  ``rms``: norms that do not subtract the mean.
    ``out`` receives the stream and may be h, ``x_out`` x and may be y.

    Returns (stream, x or None, stats); stats ([4][rows] fp32) is what
    :func:`residual_norm_backward` needs."""
    a = _residual_args(h, y, weight, bias, post_weight, post_bias, gate, alpha, rms, eps)
    dev, kind = h.device, h.dtype
    if weight is None and x_out is not None:
        raise ValueError("without weight there is no x")
    with _launch(dev, stream, h, y, weight, bias, post_weight, post_bias, gate, out, x_out) as s:
        if out is None:
            out = torch.empty(h.shape, dtype=kind, device=dev)
        os = _rows(out, "out", (kind,), dev, h.shape)[2]
        xs = 0
        if weight is not None:
            if x_out is None:
                x_out = torch.empty(h.shape, dtype=kind, device=dev)
            xs = _rows(x_out, "x_out", (kind,), dev, h.shape)[2]
        stats = torch.empty((4, a.rows), dtype=torch.float32, device=dev)
        rc = _sieve.lib().sieve_residual_norm(C.byref(a), out.data_ptr(), os, _ptr(x_out), xs, stats.data_ptr(), s)
        if rc:
            _sieve._check(rc, "sieve_residual_norm")
    return out, x_out, stats


def residual_norm_backward(dstream, dx, h, y, stats, weight=None, bias=None, post_weight=None, post_bias=None,
                           gate=None, alpha=1.0, rms=False, out=None, dy_out=None, workspace=None, stream=None):
    """Gradients of :func:`residual_norm` from those of its results
    (sieve_residual_norm_backward): ``dstream`` (None: the stream is not used
    further; needed without weight) and ``dx`` (None without weight).

    h, y and the other arguments are the forward call's, ``stats`` its result.
    ``out`` receives dh and may be dstream, ``dy_out`` dy and may be dx.
    Returns (dh, dy, dweight, dbias, dpost_weight, dpost_bias, dgate), None for
    what was not given."""
    a = _residual_args(h, y, weight, bias, post_weight, post_bias, gate, alpha, rms, 0.0)
    dev, kind = h.device, h.dtype
    if (dx is None) != (weight is None):
        raise ValueError("dx is the gradient of x, which there is with a weight alone")
    if dstream is None and weight is None:
        raise ValueError("dstream is missing")
    dss = 0 if dstream is None else _rows(dstream, "dstream", (kind,), dev, h.shape)[2]
    dxs = 0 if dx is None else _rows(dx, "dx", (kind,), dev, h.shape)[2]
    _need(stats, "stats", (torch.float32,), 2, dev)
    if tuple(stats.shape) != (4, a.rows) or not stats.is_contiguous():
        raise ValueError("stats must be the forward call's")
    lib = _sieve.lib()
    n = _size()
    _sieve._check(lib.sieve_residual_norm_backward_workspace_size(a.rows, a.width, C.byref(n)),
                  "sieve_residual_norm_backward_workspace_size")
    with _launch(dev, stream, dstream, dx, h, y, stats, weight, bias, post_weight, post_bias, gate, out, dy_out) as s:
        def like(t):
            return None if t is None else torch.empty(t.shape, dtype=t.dtype, device=dev)
        if out is None:
            out = torch.empty(h.shape, dtype=kind, device=dev)
        if dy_out is None:
            dy_out = torch.empty(h.shape, dtype=kind, device=dev)
        dhs, dys = _rows(out, "out", (kind,), dev, h.shape)[2], _rows(dy_out, "dy_out", (kind,), dev, h.shape)[2]
        grads = [like(t) for t in (weight, bias, post_weight, post_bias)]
        dgate = like(gate)
        g = ResidualNormGradsC(_ptr(dstream), _ptr(dx), dss, dxs, stats.data_ptr(), out.data_ptr(), dy_out.data_ptr(),
                               _ptr(dgate), dhs, dys, a.width, *(_ptr(t) for t in grads))
        ws = _scratch(workspace, n.value, dev)
        _sieve._check(lib.sieve_residual_norm_backward(C.byref(a), C.byref(g), ws.data_ptr(), ws.numel(), s),
                      "sieve_residual_norm_backward")
    return out, dy_out, *grads, dgate


# ---------------------------------------------------------------------------
def _loss_args(h, weight, targets, bias, scale, wait_limit):
    rows, width, hs = _tiles(h, "h", _HALVES)
    dev = h.device
    classes, w_width, ws = _tiles(weight, "weight", (h.dtype,), dev)
    if w_width != width:
        raise ValueError(f"h {tuple(h.shape)} and weight {tuple(weight.shape)} do not fit together")
    _ids(targets, "targets", dev, rows)
    if bias is not None:
        _vector(bias, "bias", (torch.float32,), classes, dev)
    return CrossEntropyArgsC(rows, classes, width, DTYPES[h.dtype], ID_TYPES[targets.dtype], scale, h.data_ptr(),
                             weight.data_ptr(), hs, ws, _ptr(bias), targets.data_ptr(), wait_limit)


def cross_entropy(h, weight, targets, bias=None, scale=1.0, workspace=None, stream=None, check=False, wait_limit=0):
    """Softmax cross entropy of the rows ``h`` [rows][width] against the
    classes ``weight`` [classes][width] (both fp16 or bf16, width a multiple
    of 8): scores scale h.weight + bias, which are not kept
    (sieve_cross_entropy).  ``bias``: [classes] fp32, -inf hides a class.

    ``targets`` (int32 or int64 [rows]): the class of each row; one outside
    [0, classes) means none, and such a row has a loss and an lse of 0 and
    costs nothing.  ``check``: read the device status afterwards (synchronizes)
    and raise if a bounded wait gave up; ``wait_limit`` shortens one of them, for
    tests of that.  Returns (loss, lse), [rows] fp32."""
    a = _loss_args(h, weight, targets, bias, scale, wait_limit)
    dev = h.device
    lib = _sieve.lib()
    n = _size()
    ref = C.byref(a)
    _sieve._check(lib.sieve_cross_entropy_workspace_size(ref, C.byref(n)), "sieve_cross_entropy_workspace_size")
    with _launch(dev, stream, h, weight, targets, bias) as s:
        loss = torch.empty(a.rows, dtype=torch.float32, device=dev)
        lse = torch.empty(a.rows, dtype=torch.float32, device=dev)
        ws = _scratch(workspace, n.value, dev)
        _sieve._check(lib.sieve_cross_entropy(ref, loss.data_ptr(), lse.data_ptr(), ws.data_ptr(), ws.numel(), s),
                      "sieve_cross_entropy")
        if check:
            _sieve._check(encoder_status(ws, s), "sieve_cross_entropy (device status)")
    return loss, lse


def cross_entropy_backward(dloss, h, weight, targets, loss, lse, bias=None, scale=1.0, dweight=None, accumulate=False,
                           need_dh=True, need_dweight=True, workspace=None, stream=None, check=False, wait_limit=0):
    """Gradients of :func:`cross_entropy` for the gradient ``dloss`` [rows]
    fp32 of every row's loss: (dh, dweight, dbias), dbias fp32 and None without
    a bias (sieve_cross_entropy_backward).

    ``loss`` and ``lse`` are the forward call's results, the other arguments the
    same as there.  ``dweight``: the tensor to write, of weight's type or
    fp32 (default: a new one of weight's type); ``accumulate`` adds to it, fp32
    alone.  Rows without a target get a dh of zero.  ``need_dh=False``,
    ``need_dweight=False``: leave the product out, None in its place."""
    a = _loss_args(h, weight, targets, bias, scale, wait_limit)
    dev = h.device
    for t, name in ((dloss, "dloss"), (loss, "loss"), (lse, "lse")):
        _vector(t, name, (torch.float32,), a.rows, dev)
    if dweight is not None and not need_dweight:
        raise ValueError("dweight is not needed")
    if accumulate and (dweight is None or dweight.dtype != torch.float32):
        raise ValueError("accumulate adds to a dweight of float32")
    lib = _sieve.lib()
    n = _size()
    ref = C.byref(a)
    _sieve._check(lib.sieve_cross_entropy_backward_workspace_size(ref, C.byref(n)),
                  "sieve_cross_entropy_backward_workspace_size")
    with _launch(dev, stream, dloss, h, weight, targets, loss, lse, bias, dweight) as s:
        dh = torch.empty(h.shape, dtype=h.dtype, device=dev) if need_dh else None
        if dweight is None and need_dweight:
            dweight = torch.empty(weight.shape, dtype=weight.dtype, device=dev)
        dws = 0 if dweight is None else _tiles(dweight, "dweight", (weight.dtype, torch.float32), dev, weight.shape)[2]
        dbias = None if bias is None else torch.empty(a.classes, dtype=torch.float32, device=dev)
        g = CrossEntropyGradsC(dloss.data_ptr(), loss.data_ptr(), lse.data_ptr(), _ptr(dh), _ptr(dweight), a.width, dws,
                               DTYPES[weight.dtype if dweight is None else dweight.dtype], 1 if accumulate else 0,
                               _ptr(dbias))
        ws = _scratch(workspace, n.value, dev)
        _sieve._check(lib.sieve_cross_entropy_backward(ref, C.byref(g), ws.data_ptr(), ws.numel(), s),
                      "sieve_cross_entropy_backward")
        if check:
            _sieve._check(encoder_status(ws, s), "sieve_cross_entropy_backward (device status)")
    return dh, dweight, dbias
