"""The model operators of include/malt.h on torch tensors: the embedding lookup and
its gradient, the norms of queries and keys with the position rotation and their
gradient, the RMS norm of a residual stream (also to 8 bits) and its gradient,
distillation from a teacher's top logits, and the cross entropy of an output head
without its logits, with its gradients.

Each function checks its tensors (ValueError for a shape, type, layout or device
that the library cannot take), allocates what it returns unless an output is
given, and enqueues the library's kernels on `stream` (default: the current one)
without synchronising.  Tensors live on the current CUDA device.  A head, and a row of
embeddings, logits or teacher's entries, is contiguous; heads may lie at any strides, rows
at one stride (those of x[..., :n] do, those of x[:, :-1] with three dimensions do not);
vectors, tables of angles and token ids are contiguous.

With a `stream` other than the current one, the caller orders its inputs and the use of
its outputs; what is allocated here belongs to that stream, and results may be dropped at
any time.

Results belong to no autograd graph, also those of tensors that require gradients: a
gradient is a call of its own (an autograd.Function calls it, as toy_distill.py does
for qk_norm and toy_language.py for rms_norm).  An output that is given counts as modified, so that a backward pass
that has kept it refuses.

For a few tokens the time of a call is the host's, so the checks read each property
of a tensor once, the current device and stream come from torch._C, without the Python
objects around them, and outputs come from the cheapest of torch's allocating calls.
"""
from __future__ import annotations

import struct

import torch

from . import malt

_FLOATS = {torch.float32: malt.MALT_F32, torch.bfloat16: malt.MALT_BF16}
_INDEX = {torch.int32: malt.MALT_I32, torch.int64: malt.MALT_I64}
# malt_embed_t, malt_qk_norm_t, malt_heads_t and malt_distill_t (native alignment)
_EMBED = struct.Struct("PiiifqqqPqPq")
_QK = struct.Struct("iiiiifqqPiiqPPqPP")
_HEADS = struct.Struct("Pqqqq")
_DISTILL = struct.Struct("PqqqiiPqPqqPif")
_RMS = struct.Struct("Pifqq")           # malt_rms_norm_t
_ROWS = struct.Struct("Pqii")           # malt_rows_t
_HEAD = struct.Struct("PqPqPPqqqiiii")  # malt_head_t


# Tells autograd that a tensor changes, for its check of what a backward pass has kept.
_written = torch.autograd.graph.increment_version
# The raw handle of a device's current stream, and the current device.
_current_stream = torch._C._cuda_getCurrentRawStream
_current_device = torch._C._cuda_getDevice


def _check(code: int, where: str):
    if code != malt.MALT_OK:
        raise malt.MaltError(code, where)


def _device(names, *tensors):
    """The current CUDA device, which all tensors (None entries aside) are on."""
    dev = tensors[0].get_device()
    for t in tensors:
        if t is not None and t.get_device() != dev:
            dev = -1
            break
    if dev < 0 or dev != _current_device():
        where = {n: str(t.device) for n, t in zip(names.split(), tensors) if t is not None}
        raise ValueError(f"tensors must be on the current CUDA device: {where}")
    return dev


def _on(stream, op, *args):
    """op(*args) with `stream` as the current one.  What the call allocates is then free for reuse
    in that stream's order; its results are kept until both streams are done with them."""
    caller = torch.cuda.current_stream()
    with torch.cuda.stream(stream):
        results = op(*args)
    for t in results if isinstance(results, tuple) else (results,):
        if t is not None:
            t.record_stream(caller)
            t.record_stream(stream)
    return results


def _float_code(name, t):
    code = _FLOATS.get(t.dtype)
    if code is None:
        raise ValueError(f"{name} must be float32 or bfloat16, not {t.dtype}")
    return code


def _index_code(name, t):
    code = _INDEX.get(t.dtype)
    if code is None:
        raise ValueError(f"{name} must be int32 or int64, not {t.dtype}")
    return code


def _row_stride(name, t, cols):
    """Elements between two rows of t seen as a matrix of its last dimension."""
    if t.is_contiguous():
        return cols
    st, shape = t.stride(), t.shape
    if cols > 1 and st[-1] != 1:
        raise ValueError(f"{name} must have contiguous rows")
    ld, after = cols, 0         # `after` rows of all the dimensions so far: the next one's stride
    for n, d in zip(shape[-2::-1], st[-2::-1]):
        if n == 1:
            continue
        if after == 0:
            ld = d
        elif d != after:
            raise ValueError(f"the rows of {name} must lie at one stride")
        after = d * n
        if ld < cols:
            raise ValueError(f"{name} has overlapping rows")
    return ld


def _vector(name, t, n, dtypes=(torch.float32,)):
    if t is not None and (t.numel() != n or t.dtype not in dtypes or not t.is_contiguous()):
        raise ValueError(f"{name} must be a contiguous vector of {n} entries of {dtypes}")


def _pointer(t):
    return 0 if t is None else t.data_ptr()


# ---------------------------------------------------------------- embedding

def embed(table, ids, scale: float = 1.0, dtype=None, out=None, stream=None):
    """scale * table[ids], of shape ids.shape + (dim,) in `dtype` (default: the
    table's).  A negative id is padding (a zero row); an id past the table gives
    a NaN row.  ids must be contiguous."""
    if stream is not None:
        return _on(stream, embed, table, ids, scale, dtype, out)
    dev = _device("table ids out", table, ids, out)
    if table.dim() != 2:
        raise ValueError("table must be a vocab x dim matrix")
    if not ids.is_contiguous():
        raise ValueError("ids must be contiguous")
    vocab, dim = table.shape
    shape = (*ids.shape, dim)
    if out is None:
        out = torch.empty(shape, dtype=table.dtype if dtype is None else dtype, device=table.device)
    elif out.shape != shape or dtype not in (None, out.dtype):
        raise ValueError(f"out has shape {tuple(out.shape)} and dtype {out.dtype}, expected {shape} and {dtype}")
    else:
        _written(out)
    e = _EMBED.pack(ids.data_ptr(), _index_code("ids", ids), _float_code("table", table), _float_code("out", out),
                    scale, ids.numel(), vocab, dim, table.data_ptr(), _row_stride("table", table, dim),
                    out.data_ptr(), _row_stride("out", out, dim))
    _check(malt.load().malt_embed_forward(e, _current_stream(dev)), "malt_embed_forward")
    return out


def embed_grad(dout, ids, vocab: int, scale: float = 1.0, dtype=None, out=None, accumulate: bool = False,
               stream=None):
    """The gradient of embed's table: row v is scale times the sum of dout's rows whose
    id is v.  Returns a vocab x dim matrix in `dtype` (default: float32), every row
    written; with `accumulate` the sums are added to `out` instead (only rows that
    occur are touched).  ids must be contiguous."""
    if stream is not None:
        return _on(stream, embed_grad, dout, ids, vocab, scale, dtype, out, accumulate)
    dev = _device("dout ids out", dout, ids, out)
    if not ids.is_contiguous():
        raise ValueError("ids must be contiguous")
    if dout.dim() < 1 or dout.shape[:-1] != ids.shape:
        raise ValueError(f"dout has shape {tuple(dout.shape)}, expected {tuple(ids.shape)} + (dim,)")
    dim = dout.shape[-1]
    if out is None:
        if accumulate:
            raise ValueError("accumulate needs the matrix to add to (out)")
        out = torch.empty((vocab, dim), dtype=torch.float32 if dtype is None else dtype, device=dout.device)
    elif out.shape != (vocab, dim) or dtype not in (None, out.dtype):
        raise ValueError(f"out has shape {tuple(out.shape)} and dtype {out.dtype}, expected {(vocab, dim)} and {dtype}")
    else:
        _written(out)
    lib = malt.load()
    n = ids.numel()
    size = lib.malt_embed_workspace_bytes(n, dim)
    ws = torch.empty(size, dtype=torch.uint8, device=dout.device)
    e = _EMBED.pack(ids.data_ptr(), _index_code("ids", ids), _float_code("out", out), _float_code("dout", dout),
                    scale, n, vocab, dim, out.data_ptr(), _row_stride("out", out, dim),
                    dout.data_ptr(), _row_stride("dout", dout, dim))
    _check(lib.malt_embed_backward(e, 1 if accumulate else 0, ws.data_ptr(), size, _current_stream(dev)),
           "malt_embed_backward")
    return out


# ------------------------------------------------- norms of queries and keys

def _like(name, t, like):
    """t, given for something of like's shape and dtype, or memory for it."""
    if t is None:
        return torch.empty_like(like)
    if t.shape != like.shape or t.dtype != like.dtype:
        raise ValueError(f"{name} has shape {tuple(t.shape)} and dtype {t.dtype}, expected {tuple(like.shape)} "
                         f"and {like.dtype}")
    if 0 in t.stride() and not t.is_contiguous():
        raise ValueError(f"{name} has overlapping entries")
    _written(t)
    return t


def _heads(t):
    """malt_heads_t of a [batch, seq, heads, dim] or [tokens, heads, dim] tensor."""
    st, shape = t.stride(), t.shape
    if st[-1] != 1 and shape[-1] > 1:
        raise ValueError("the entries of a head must be contiguous")
    if len(st) == 4:
        return _HEADS.pack(t.data_ptr(), shape[2], st[0], st[1], st[2])
    return _HEADS.pack(t.data_ptr(), shape[1], 0, st[0], st[1])


def _qk_params(q, k, q_gain, k_gain, cos, sin, positions, eps, interleaved):
    shape, k_shape = q.shape, k.shape
    rank, dim = len(shape), shape[-1]
    if rank not in (3, 4) or len(k_shape) != rank:
        raise ValueError("q and k must be [batch, seq, heads, dim] or [tokens, heads, dim] tensors")
    if k_shape[:-2] != shape[:-2] or k_shape[-1] != dim or k.dtype != q.dtype:
        raise ValueError(f"q {tuple(shape)} {q.dtype} and k {tuple(k_shape)} {k.dtype} differ in more than heads")
    batch, seq = (1, shape[0]) if rank == 3 else shape[:2]
    rows, pairs = cos.shape if cos.dim() == 2 else (0, -1)
    if (pairs < 0 or cos.shape != sin.shape or cos.dtype != torch.float32 or sin.dtype != torch.float32
            or not cos.is_contiguous() or not sin.is_contiguous()):
        raise ValueError("cos and sin must be contiguous float32 matrices of one shape")
    gain_type = malt.MALT_F32
    for name, g in (("q_gain", q_gain), ("k_gain", k_gain)):
        if g is not None:
            gain_type = _float_code(name, g)
            if g.numel() != dim or not g.is_contiguous():
                raise ValueError(f"{name} must be a contiguous vector of {dim} entries")
    if q_gain is not None and k_gain is not None and q_gain.dtype != k_gain.dtype:
        raise ValueError("q_gain and k_gain must have one dtype")
    stride = index = 0
    if positions is not None:
        index = _index_code("positions", positions)
        p_shape, p_stride = positions.shape, positions.stride()
        if p_shape == (batch, seq):
            stride = p_stride[0]
        elif p_shape != (seq,):
            raise ValueError(f"positions has shape {tuple(p_shape)}, expected {(batch, seq)} or {(seq,)}")
        if seq > 1 and p_stride[-1] != 1:
            raise ValueError("the last dimension of positions must be contiguous")
    return _QK.pack(_float_code("q", q), gain_type, dim, 2 * pairs, 1 if interleaved else 0, eps, batch, seq,
                    _pointer(positions), index, 0, stride, cos.data_ptr(), sin.data_ptr(), rows,
                    _pointer(q_gain), _pointer(k_gain))


def qk_norm(q, k, q_gain, k_gain, cos, sin, positions=None, eps: float = 1e-6, interleaved: bool = False,
            q_out=None, k_out=None, stream=None):
    """Every head of q and k divided by its root mean square and multiplied by its gain (None:
    ones), its first 2 * cos.shape[1] entries rotated by the angles of the token's position.

    q, k: [batch, seq, heads, dim] or [tokens, heads, dim], any strides before the last
    dimension; cos, sin: [positions, pairs]; positions: [batch, seq] or [seq] ([tokens]),
    default 0 .. seq-1.  Pairs are (i, pairs + i), or (2i, 2i+1) when interleaved.
    Returns (q_out, k_out); each may be given, also as its input itself."""
    if stream is not None:
        return _on(stream, qk_norm, q, k, q_gain, k_gain, cos, sin, positions, eps, interleaved, q_out, k_out)
    dev = _device("q k q_gain k_gain cos sin positions q_out k_out", q, k, q_gain, k_gain, cos, sin, positions, q_out,
                  k_out)
    p = _qk_params(q, k, q_gain, k_gain, cos, sin, positions, eps, interleaved)
    q_out, k_out = _like("q_out", q_out, q), _like("k_out", k_out, k)
    _check(malt.load().malt_qk_norm_forward(p, _heads(q), _heads(k), _heads(q_out), _heads(k_out),
                                            _current_stream(dev)), "malt_qk_norm_forward")
    return q_out, k_out


def qk_norm_grad(dq_out, dk_out, q, k, q_gain, k_gain, cos, sin, positions=None, eps: float = 1e-6,
                 interleaved: bool = False, dq=None, dk=None, stream=None):
    """The gradient of qk_norm from those of its outputs and its own arguments.  Returns
    (dq, dk, dq_gain, dk_gain), the gains' gradients in float32 (None for a gain that is None); dq
    and dk may be given, also as dq_out and dk_out themselves."""
    if stream is not None:
        return _on(stream, qk_norm_grad, dq_out, dk_out, q, k, q_gain, k_gain, cos, sin, positions, eps, interleaved,
                   dq, dk)
    dev = _device("q k dq_out dk_out q_gain k_gain cos sin positions dq dk", q, k, dq_out, dk_out, q_gain, k_gain, cos,
                  sin, positions, dq, dk)
    p = _qk_params(q, k, q_gain, k_gain, cos, sin, positions, eps, interleaved)
    if dq_out.shape != q.shape or dk_out.shape != k.shape or dq_out.dtype != q.dtype or dk_out.dtype != k.dtype:
        raise ValueError("dq_out and dk_out must have the shapes and dtype of q and k")
    dq, dk = _like("dq", dq, q), _like("dk", dk, k)
    dim = q.shape[-1]
    dq_gain = None if q_gain is None else torch.empty(dim, dtype=torch.float32, device=q.device)
    dk_gain = None if k_gain is None else torch.empty(dim, dtype=torch.float32, device=q.device)
    lib = malt.load()
    size = lib.malt_qk_norm_workspace_bytes(dim)
    ws = torch.empty(size, dtype=torch.uint8, device=q.device)
    _check(lib.malt_qk_norm_backward(p, _heads(dq_out), _heads(dk_out), _heads(q), _heads(k), _heads(dq), _heads(dk),
                                     _pointer(dq_gain), _pointer(dk_gain), ws.data_ptr(), size,
                                     _current_stream(dev)), "malt_qk_norm_backward")
    return dq, dk, dq_gain, dk_gain


# ------------------------------------------------ norm of a residual stream

NORM_GROUP = 128        # entries of a row that share a scale in 8 bits


def _rows(name, t, dim, dtype=None):
    """malt_rows_t of a tensor seen as a matrix of its last dimension."""
    return _ROWS.pack(t.data_ptr(), _row_stride(name, t, dim), _float_code(name, t) if dtype is None else dtype, 0)


def _rms_params(like, gain, eps):
    if like.dim() < 1 or like.shape[-1] < 1:
        raise ValueError("rows must have entries")
    dim = like.shape[-1]
    if gain is not None:
        _vector("gain", gain, dim, tuple(_FLOATS))
    return _RMS.pack(_pointer(gain), 0 if gain is None else _FLOATS[gain.dtype], eps, like.numel() // dim, dim), dim


def _same_shape(name, t, like, dtype=None):
    if t.shape != like.shape or dtype not in (None, t.dtype):
        raise ValueError(f"{name} has shape {tuple(t.shape)} and dtype {t.dtype}, expected {tuple(like.shape)}"
                         + (f" and {dtype}" if dtype is not None else ""))


def _stream_sum(x, residual, residual_out):
    """The tensor that takes x + residual, None without a stream."""
    if residual is None:
        if residual_out is not None:
            raise ValueError("residual_out needs a residual")
        return None
    _same_shape("residual", residual, x)
    if residual_out is None:
        return torch.empty_like(residual)
    _same_shape("residual_out", residual_out, x, residual.dtype)
    _written(residual_out)
    return residual_out


def rms_norm(x, gain, residual=None, eps: float = 1e-6, dtype=None, out=None, residual_out=None, stream=None):
    """(y, h): h = x + residual, rounded to the residual's type (x itself without one), and every row
    of h divided by its root mean square and multiplied by gain (None: ones), in `dtype` (default:
    x's).  out (y) and residual_out (h) may be given, each also as x or the residual
    (its type and layout), not both as one, and else apart from them (with out=x and no
    residual x is y, and no h is left for the gradient)."""
    if stream is not None:
        return _on(stream, rms_norm, x, gain, residual, eps, dtype, out, residual_out)
    dev = _device("x gain residual out residual_out", x, gain, residual, out, residual_out)
    p, dim = _rms_params(x, gain, eps)
    h = _stream_sum(x, residual, residual_out)
    if out is None:
        out = torch.empty_like(x) if dtype in (None, x.dtype) else torch.empty(x.shape, dtype=dtype, device=x.device)
    else:
        _same_shape("out", out, x, dtype)
        _written(out)
    _check(malt.load().malt_rms_norm_forward(
        p, _rows("x", x, dim), None if h is None else _rows("residual", residual, dim),
        None if h is None else _rows("residual_out", h, dim), _rows("out", out, dim), _current_stream(dev)),
        "malt_rms_norm_forward")
    return out, x if h is None else h


def rms_norm_8bit(x, gain, residual=None, eps: float = 1e-6, out=None, residual_out=None, stream=None):
    """rms_norm with y in 8 bits: (codes, scales, h), codes float8_e4m3fn of x's shape, and a float32
    scale for every 128 entries of a row (the last may cover fewer): y is codes times scales."""
    if stream is not None:
        return _on(stream, rms_norm_8bit, x, gain, residual, eps, out, residual_out)
    dev = _device("x gain residual out residual_out", x, gain, residual, out, residual_out)
    p, dim = _rms_params(x, gain, eps)
    h = _stream_sum(x, residual, residual_out)
    if out is None:
        out = torch.empty(x.shape, dtype=torch.float8_e4m3fn, device=x.device)
    else:
        _same_shape("out", out, x, torch.float8_e4m3fn)
        _written(out)
    groups = -(-dim // NORM_GROUP)
    scales = torch.empty((*x.shape[:-1], groups), dtype=torch.float32, device=x.device)
    _check(malt.load().malt_rms_norm_forward_8bit(
        p, _rows("x", x, dim), None if h is None else _rows("residual", residual, dim),
        None if h is None else _rows("residual_out", h, dim), _rows("out", out, dim, malt.MALT_E4M3),
        scales.data_ptr(), groups, _current_stream(dev)), "malt_rms_norm_forward_8bit")
    return out, scales, x if h is None else h


def rms_norm_grad(dy, h, gain, dh=None, eps: float = 1e-6, out=None, stream=None):
    """The gradient of rms_norm from that of y and the h that it returned: (dx, dgain), dx the gradient
    of x and of the residual alike, with dh (the gradient that reaches h from the stream) added, in
    h's type, and dgain in float32 (None for a gain that is None).  out (dx) may be given, also as dy,
    h or dh."""
    if stream is not None:
        return _on(stream, rms_norm_grad, dy, h, gain, dh, eps, out)
    dev = _device("h dy gain dh out", h, dy, gain, dh, out)
    p, dim = _rms_params(h, gain, eps)
    _same_shape("dy", dy, h)
    if dh is not None:
        _same_shape("dh", dh, h, h.dtype)
    if out is None:
        out = torch.empty_like(h)
    else:
        _same_shape("out", out, h, h.dtype)
        _written(out)
    dgain, ws, size = None, None, 0
    lib = malt.load()
    if gain is not None:
        dgain = torch.empty(dim, dtype=torch.float32, device=h.device)
        size = lib.malt_rms_norm_workspace_bytes(h.numel() // dim, dim)
        ws = torch.empty(size, dtype=torch.uint8, device=h.device)
    _check(lib.malt_rms_norm_backward(p, _rows("dy", dy, dim), _rows("h", h, dim),
                                      None if dh is None else _rows("dh", dh, dim), _rows("out", out, dim),
                                      _pointer(dgain), _pointer(ws), size, _current_stream(dev)),
           "malt_rms_norm_backward")
    return out, dgain


# -------------------------------------------------------------- distillation

def _distill_params(logits, top_ids, top_logits, weight, temperature):
    vocab = logits.shape[-1]
    rows = logits.numel() // max(vocab, 1)
    if top_ids.shape != top_logits.shape or top_ids.shape[:-1] != logits.shape[:-1]:
        raise ValueError(f"top_ids {tuple(top_ids.shape)} and top_logits {tuple(top_logits.shape)} must have the rows "
                         f"of logits {tuple(logits.shape)}")
    _vector("weight", weight, rows)
    top = top_ids.shape[-1]
    return _DISTILL.pack(logits.data_ptr(), _row_stride("logits", logits, vocab), rows, vocab,
                         _float_code("logits", logits), _index_code("top_ids", top_ids), top_ids.data_ptr(),
                         _row_stride("top_ids", top_ids, top), top_logits.data_ptr(),
                         _row_stride("top_logits", top_logits, top), top, _pointer(weight),
                         _float_code("top_logits", top_logits), temperature)


def _loss(logits):
    return torch.empty(logits.shape[:-1], dtype=torch.float32, device=logits.device)


def distill_loss(logits, top_ids, top_logits, weight=None, temperature: float = 1.0, stream=None):
    """Per row, weight * T^2 * KL(p || q) of the teacher's distribution p over its listed
    entries (top_ids, top_logits) and the student's q over the vocabulary, both at temperature T.
    Returns (loss, stats): float32 losses of shape logits.shape[:-1], and the row
    statistics [rows, 2] that distill_grad takes.  Entries with an id outside the
    vocabulary or a logit of -inf are not listed; rows of weight 0 or with nothing
    listed have loss 0."""
    if stream is not None:
        return _on(stream, distill_loss, logits, top_ids, top_logits, weight, temperature)
    dev = _device("logits top_ids top_logits weight", logits, top_ids, top_logits, weight)
    d = _distill_params(logits, top_ids, top_logits, weight, temperature)
    loss = _loss(logits)
    stats = torch.empty((loss.numel(), 2), dtype=torch.float32, device=logits.device)
    _check(malt.load().malt_distill_forward(d, loss.data_ptr(), stats.data_ptr(), _current_stream(dev)),
           "malt_distill_forward")
    return loss, stats


def distill_grad(logits, top_ids, top_logits, stats, dloss=None, weight=None, temperature: float = 1.0,
                 dlogits=None, stream=None):
    """The gradient of the logits from distill_loss's statistics and the gradient of each row's
    loss (None: ones), in the logits' type; dlogits may be given, also as the logits."""
    if stream is not None:
        return _on(stream, distill_grad, logits, top_ids, top_logits, stats, dloss, weight, temperature, dlogits)
    dev = _device("logits top_ids top_logits weight stats dloss dlogits", logits, top_ids, top_logits, weight, stats,
                  dloss, dlogits)
    d = _distill_params(logits, top_ids, top_logits, weight, temperature)
    rows = logits.numel() // max(logits.shape[-1], 1)
    _vector("stats", stats, 2 * rows)
    _vector("dloss", dloss, rows)
    dlogits = _like("dlogits", dlogits, logits)
    ld = _row_stride("dlogits", dlogits, logits.shape[-1])
    _check(malt.load().malt_distill_backward(d, stats.data_ptr(), _pointer(dloss), dlogits.data_ptr(), ld,
                                             _current_stream(dev)), "malt_distill_backward")
    return dlogits


def distill_loss_grad(logits, top_ids, top_logits, weight=None, temperature: float = 1.0, dlogits=None, stream=None):
    """distill_loss and the gradient of the losses' sum in one pass over the logits (a mean is a
    weight of 1 / rows).  Returns (loss, dlogits); dlogits may be given, also as the logits."""
    if stream is not None:
        return _on(stream, distill_loss_grad, logits, top_ids, top_logits, weight, temperature, dlogits)
    dev = _device("logits top_ids top_logits weight dlogits", logits, top_ids, top_logits, weight, dlogits)
    d = _distill_params(logits, top_ids, top_logits, weight, temperature)
    loss = _loss(logits)
    dlogits = _like("dlogits", dlogits, logits)
    ld = _row_stride("dlogits", dlogits, logits.shape[-1])
    _check(malt.load().malt_distill_forward_backward(d, loss.data_ptr(), 0, dlogits.data_ptr(), ld,
                                                     _current_stream(dev)), "malt_distill_forward_backward")
    return loss, dlogits


# ------------------------------------------------- cross entropy of an output head

def _head_params(hidden, table, labels, weight):
    """(malt_head_t, rows)."""
    if table.dim() != 2 or hidden.dim() < 1 or hidden.shape[-1] != table.shape[1]:
        raise ValueError(f"hidden {tuple(hidden.shape)} and table {tuple(table.shape)} must have rows of one length")
    vocab, dim = table.shape
    if vocab < 1 or dim < 1:
        raise ValueError("table must have entries")
    if labels.shape != hidden.shape[:-1] or not labels.is_contiguous():
        raise ValueError(f"labels must be contiguous, of shape {tuple(hidden.shape[:-1])}")
    rows = labels.numel()
    _vector("weight", weight, rows)
    return _HEAD.pack(hidden.data_ptr(), _row_stride("hidden", hidden, dim), table.data_ptr(),
                      _row_stride("table", table, dim), labels.data_ptr(), _pointer(weight), rows, dim, vocab,
                      _float_code("hidden", hidden), _float_code("table", table), _index_code("labels", labels), 0), rows


def _head_workspace(lib, h, forward, gradient, like):
    size = lib.malt_head_workspace_bytes(h, forward, gradient)
    if size == 0:
        raise ValueError("sizes past the limits of the head's operators")
    return torch.empty(size, dtype=torch.uint8, device=like.device), size


def _head_gradients(hidden, table, dhidden, dtable, dtype, accumulate):
    if dtable is None:
        if accumulate:
            raise ValueError("accumulate needs the matrix to add to (dtable)")
        dtable = torch.empty(table.shape, dtype=table.dtype if dtype is None else dtype, device=table.device)
    else:
        _same_shape("dtable", dtable, table, dtype)
        _written(dtable)
    if dhidden is None:
        dhidden = torch.empty(hidden.shape, dtype=hidden.dtype, device=hidden.device)
    else:
        _same_shape("dhidden", dhidden, hidden, hidden.dtype)
        _written(dhidden)
    return dhidden, dtable


def _head_outputs(dhidden, dtable, accumulate):
    return (dhidden.data_ptr(), _row_stride("dhidden", dhidden, dhidden.shape[-1]), dtable.data_ptr(),
            _row_stride("dtable", dtable, dtable.shape[1]), _float_code("dtable", dtable), 1 if accumulate else 0)


def head_loss(hidden, table, labels, weight=None, stream=None):
    """Per row, weight times the cross entropy of softmax(hidden @ table.T) and the label, without keeping the
    logits.  Returns (loss, stats): float32 losses of labels' shape, and the row statistics [rows, 2] (maximum
    and sum of exponentials) that head_grad takes.  Rows with a negative label or weight 0 have loss 0;
    a label past the table has loss NaN."""
    if stream is not None:
        return _on(stream, head_loss, hidden, table, labels, weight)
    dev = _device("hidden table labels weight", hidden, table, labels, weight)
    h, rows = _head_params(hidden, table, labels, weight)
    lib = malt.load()
    ws, size = _head_workspace(lib, h, 1, 0, hidden)
    loss = torch.empty(labels.shape, dtype=torch.float32, device=hidden.device)
    stats = torch.empty((rows, 2), dtype=torch.float32, device=hidden.device)
    _check(lib.malt_head_forward(h, loss.data_ptr(), stats.data_ptr(), ws.data_ptr(), size, _current_stream(dev)),
           "malt_head_forward")
    return loss, stats


def head_grad(hidden, table, labels, stats, dloss=None, weight=None, dhidden=None, dtable=None, dtype=None,
              accumulate: bool = False, stream=None):
    """(dhidden, dtable) from head_loss's statistics and the gradient of each row's loss (None: ones): dhidden in
    hidden's type, dtable in `dtype` (default: the table's), or added to what the given dtable holds with
    `accumulate`.  Both may be given."""
    if stream is not None:
        return _on(stream, head_grad, hidden, table, labels, stats, dloss, weight, dhidden, dtable, dtype, accumulate)
    dev = _device("hidden table labels weight stats dloss dhidden dtable", hidden, table, labels, weight, stats, dloss,
                  dhidden, dtable)
    h, rows = _head_params(hidden, table, labels, weight)
    _vector("stats", stats, 2 * rows)
    _vector("dloss", dloss, rows)
    dhidden, dtable = _head_gradients(hidden, table, dhidden, dtable, dtype, accumulate)
    lib = malt.load()
    ws, size = _head_workspace(lib, h, 0, 1, hidden)
    _check(lib.malt_head_backward(h, stats.data_ptr(), _pointer(dloss), *_head_outputs(dhidden, dtable, accumulate),
                                  ws.data_ptr(), size, _current_stream(dev)), "malt_head_backward")
    return dhidden, dtable


def head_loss_grad(hidden, table, labels, weight=None, dhidden=None, dtable=None, dtype=None, accumulate: bool = False,
                   stream=None):
    """head_loss and the gradients of the losses' sum (a mean is a weight of 1 / rows).  Returns
    (loss, dhidden, dtable), as head_loss and head_grad do."""
    if stream is not None:
        return _on(stream, head_loss_grad, hidden, table, labels, weight, dhidden, dtable, dtype, accumulate)
    dev = _device("hidden table labels weight dhidden dtable", hidden, table, labels, weight, dhidden, dtable)
    h, rows = _head_params(hidden, table, labels, weight)
    dhidden, dtable = _head_gradients(hidden, table, dhidden, dtable, dtype, accumulate)
    lib = malt.load()
    ws, size = _head_workspace(lib, h, 1, 1, hidden)
    loss = torch.empty(labels.shape, dtype=torch.float32, device=hidden.device)
    _check(lib.malt_head_forward_backward(h, loss.data_ptr(), 0, *_head_outputs(dhidden, dtable, accumulate),
                                          ws.data_ptr(), size, _current_stream(dev)), "malt_head_forward_backward")
    return loss, dhidden, dtable
