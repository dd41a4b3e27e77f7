"""The model operators of include/malt.h on torch tensors: the embedding lookup and
its gradient, the norms of queries and keys with the position rotation and their
gradient, and distillation from a teacher's top logits.

Each function checks its tensors (ValueError for a shape, type, layout or device
that the library cannot take), allocates what it returns unless an output is
given, and enqueues the library's kernels on `stream` (default: the current one)
without synchronising.  Tensors live on the current CUDA device; only the last
dimension has to be contiguous where nothing else is said.  With a `stream` other
than the current one, the caller orders its inputs and the use of its outputs; memory
allocated here is marked as used on that stream.
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


def _check(code: int, where: str):
    if code != malt.MALT_OK:
        raise malt.MaltError(code, where)


def _on_device(**tensors):
    """The tensors (None entries aside) are CUDA tensors of the current device."""
    for name, t in tensors.items():
        if t is not None and not t.is_cuda:
            raise ValueError(f"{name} must be a CUDA tensor, not on {t.device}")
    dev = torch.cuda.current_device()
    for name, t in tensors.items():
        if t is not None and t.get_device() != dev:
            raise ValueError(f"{name} must be on the current CUDA device (cuda:{dev}), not {t.device}")


def _stream(stream, *allocated):
    """The raw stream; memory allocated for this call is kept for it."""
    current = torch.cuda.current_stream()
    if stream is None or stream == current:
        return current.cuda_stream
    for t in allocated:
        if t is not None:
            t.record_stream(stream)
    return stream.cuda_stream


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
    if t.dim() != 2 or (cols > 1 and t.stride(1) != 1):
        raise ValueError(f"{name} must be contiguous, or 2-D with contiguous rows")
    if t.shape[0] <= 1:
        return cols
    if t.stride(0) < cols:
        raise ValueError(f"{name} has overlapping rows")
    return t.stride(0)


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
    _on_device(table=table, ids=ids, out=out)
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
    e = _EMBED.pack(ids.data_ptr(), _index_code("ids", ids), _float_code("table", table), _float_code("out", out),
                    scale, ids.numel(), vocab, dim, table.data_ptr(), _row_stride("table", table, dim),
                    out.data_ptr(), _row_stride("out", out, dim))
    _check(malt.load().malt_embed_forward(e, _stream(stream, out)), "malt_embed_forward")
    return out


def embed_grad(dout, ids, vocab: int, scale: float = 1.0, dtype=None, out=None, accumulate: bool = False,
               stream=None):
    """The gradient of embed's table: row v is scale times the sum of dout's rows whose
    id is v.  Returns a vocab x dim matrix in `dtype` (default: float32), every row
    written; with `accumulate` the sums are added to `out` instead (only rows that
    occur are touched)."""
    _on_device(dout=dout, ids=ids, out=out)
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
    lib = malt.load()
    n = ids.numel()
    size = lib.malt_embed_workspace_bytes(n, dim)
    ws = torch.empty(size, dtype=torch.uint8, device=dout.device)
    e = _EMBED.pack(ids.data_ptr(), _index_code("ids", ids), _float_code("out", out), _float_code("dout", dout),
                    scale, n, vocab, dim, out.data_ptr(), _row_stride("out", out, dim),
                    dout.data_ptr(), _row_stride("dout", dout, dim))
    _check(lib.malt_embed_backward(e, 1 if accumulate else 0, ws.data_ptr(), size, _stream(stream, out, ws)),
           "malt_embed_backward")
    return out


# ------------------------------------------------- norms of queries and keys

def _heads(name, t, like=None):
    """malt_heads_t of a [batch, seq, heads, dim] or [tokens, heads, dim] tensor."""
    if like is not None and (t.shape != like.shape or t.dtype != like.dtype):
        raise ValueError(f"{name} has shape {tuple(t.shape)} and dtype {t.dtype}, expected {tuple(like.shape)} "
                         f"and {like.dtype}")
    st = t.stride()
    if st[-1] != 1 and t.shape[-1] > 1:
        raise ValueError(f"the heads of {name} must be contiguous")
    return _HEADS.pack(t.data_ptr(), t.shape[-2], st[0] if len(st) == 4 else 0, st[-3], st[-2])


def _qk_params(q, k, q_gain, k_gain, cos, sin, positions, eps, interleaved):
    if q.dim() not in (3, 4) or k.dim() != q.dim():
        raise ValueError("q and k must be [batch, seq, heads, dim] or [tokens, heads, dim] tensors")
    dim = q.shape[-1]
    if k.shape[:-2] != q.shape[:-2] or k.shape[-1] != dim or k.dtype != q.dtype:
        raise ValueError(f"q {tuple(q.shape)} {q.dtype} and k {tuple(k.shape)} {k.dtype} differ in more than heads")
    batch, seq = (1, q.shape[0]) if q.dim() == 3 else q.shape[:2]
    if (cos.dim() != 2 or cos.shape != sin.shape or cos.dtype != torch.float32 or sin.dtype != torch.float32
            or not cos.is_contiguous() or not sin.is_contiguous()):
        raise ValueError("cos and sin must be contiguous float32 matrices of one shape")
    gain_type = malt.MALT_F32
    for name, g in (("q_gain", q_gain), ("k_gain", k_gain)):
        _vector(name, g, dim, tuple(_FLOATS))
        if g is not None:
            gain_type = _FLOATS[g.dtype]
    if q_gain is not None and k_gain is not None and q_gain.dtype != k_gain.dtype:
        raise ValueError("q_gain and k_gain must have one dtype")
    stride = index = 0
    if positions is not None:
        index = _index_code("positions", positions)
        if positions.shape == (batch, seq) and positions.dim() == 2:
            stride = positions.stride(0)
        elif positions.shape != (seq,):
            raise ValueError(f"positions has shape {tuple(positions.shape)}, expected {(batch, seq)} or {(seq,)}")
        if seq > 1 and positions.stride(-1) != 1:
            raise ValueError("the last dimension of positions must be contiguous")
    return _QK.pack(_float_code("q", q), gain_type, dim, 2 * cos.shape[1], 1 if interleaved else 0, eps, batch, seq,
                    _pointer(positions), index, 0, stride, cos.data_ptr(), sin.data_ptr(), cos.shape[0],
                    _pointer(q_gain), _pointer(k_gain))


def qk_norm(q, k, q_gain, k_gain, cos, sin, positions=None, eps: float = 1e-6, interleaved: bool = False,
            q_out=None, k_out=None, stream=None):
    """Every head of q and k divided by its root mean square and multiplied by its gain (None:
    ones), its first 2 * cos.shape[1] entries rotated by the angles of the token's position.

    q, k: [batch, seq, heads, dim] or [tokens, heads, dim], any strides before the last
    dimension; cos, sin: [positions, pairs]; positions: [batch, seq] or [seq] ([tokens]),
    default 0 .. seq-1.  Pairs are (i, pairs + i), or (2i, 2i+1) when interleaved.
    Returns (q_out, k_out); each may be given, also as its input itself."""
    _on_device(q=q, k=k, q_gain=q_gain, k_gain=k_gain, cos=cos, sin=sin, positions=positions, q_out=q_out, k_out=k_out)
    p = _qk_params(q, k, q_gain, k_gain, cos, sin, positions, eps, interleaved)
    q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device) if q_out is None else q_out
    k_out = torch.empty(k.shape, dtype=k.dtype, device=k.device) if k_out is None else k_out
    _check(malt.load().malt_qk_norm_forward(p, _heads("q", q), _heads("k", k), _heads("q_out", q_out, q),
                                            _heads("k_out", k_out, k), _stream(stream, q_out, k_out)),
           "malt_qk_norm_forward")
    return q_out, k_out


def qk_norm_grad(dq_out, dk_out, q, k, q_gain, k_gain, cos, sin, positions=None, eps: float = 1e-6,
                 interleaved: bool = False, dq=None, dk=None, stream=None):
    """The gradient of qk_norm from those of its outputs and its own arguments.  Returns
    (dq, dk, dq_gain, dk_gain), the gains' gradients in float32 (None for a gain that is None); dq
    and dk may be given, also as dq_out and dk_out themselves."""
    _on_device(dq_out=dq_out, dk_out=dk_out, q=q, k=k, q_gain=q_gain, k_gain=k_gain, cos=cos, sin=sin,
               positions=positions, dq=dq, dk=dk)
    p = _qk_params(q, k, q_gain, k_gain, cos, sin, positions, eps, interleaved)
    dq = torch.empty(q.shape, dtype=q.dtype, device=q.device) if dq is None else dq
    dk = torch.empty(k.shape, dtype=k.dtype, device=k.device) if dk is None else dk
    dim = q.shape[-1]
    dq_gain = None if q_gain is None else torch.empty(dim, dtype=torch.float32, device=q.device)
    dk_gain = None if k_gain is None else torch.empty(dim, dtype=torch.float32, device=q.device)
    lib = malt.load()
    size = lib.malt_qk_norm_workspace_bytes(dim)
    ws = torch.empty(size, dtype=torch.uint8, device=q.device)
    _check(lib.malt_qk_norm_backward(p, _heads("dq_out", dq_out, q), _heads("dk_out", dk_out, k), _heads("q", q),
                                     _heads("k", k), _heads("dq", dq, q), _heads("dk", dk, k), _pointer(dq_gain),
                                     _pointer(dk_gain), ws.data_ptr(), size,
                                     _stream(stream, dq, dk, dq_gain, dk_gain, ws)), "malt_qk_norm_backward")
    return dq, dk, dq_gain, dk_gain


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


def _dlogits(logits, dlogits):
    if dlogits is None:
        dlogits = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
    elif dlogits.shape != logits.shape or dlogits.dtype != logits.dtype:
        raise ValueError(f"dlogits has shape {tuple(dlogits.shape)} and dtype {dlogits.dtype}, expected those of logits")
    return dlogits, _row_stride("dlogits", dlogits, logits.shape[-1])


def distill_loss(logits, top_ids, top_logits, weight=None, temperature: float = 1.0, stream=None):
    """Per row, weight * T^2 * KL(p || q) of the teacher's distribution p over its listed
    entries (top_ids, top_logits) and the student's q over the vocabulary, both at temperature T.
    Returns (loss, stats): float32 losses of shape logits.shape[:-1], and the row
    statistics [rows, 2] that distill_grad takes.  Entries with an id outside the
    vocabulary or a logit of -inf are not listed; rows of weight 0 or with nothing
    listed have loss 0."""
    _on_device(logits=logits, top_ids=top_ids, top_logits=top_logits, weight=weight)
    d = _distill_params(logits, top_ids, top_logits, weight, temperature)
    loss = torch.empty(logits.shape[:-1], dtype=torch.float32, device=logits.device)
    stats = torch.empty((loss.numel(), 2), dtype=torch.float32, device=logits.device)
    _check(malt.load().malt_distill_forward(d, loss.data_ptr(), stats.data_ptr(), _stream(stream, loss, stats)),
           "malt_distill_forward")
    return loss, stats


def distill_grad(logits, top_ids, top_logits, stats, dloss=None, weight=None, temperature: float = 1.0,
                 dlogits=None, stream=None):
    """The gradient of the logits from distill_loss's statistics and the gradient of each row's
    loss (None: ones), in the logits' type; dlogits may be given, also as the logits."""
    _on_device(logits=logits, top_ids=top_ids, top_logits=top_logits, weight=weight, stats=stats, dloss=dloss,
               dlogits=dlogits)
    d = _distill_params(logits, top_ids, top_logits, weight, temperature)
    rows = logits.numel() // max(logits.shape[-1], 1)
    _vector("stats", stats, 2 * rows)
    _vector("dloss", dloss, rows)
    dlogits, ld = _dlogits(logits, dlogits)
    _check(malt.load().malt_distill_backward(d, stats.data_ptr(), _pointer(dloss), dlogits.data_ptr(), ld,
                                             _stream(stream, dlogits)), "malt_distill_backward")
    return dlogits


def distill_loss_grad(logits, top_ids, top_logits, weight=None, temperature: float = 1.0, dlogits=None, stream=None):
    """distill_loss and the gradient of the losses' sum in one pass over the logits (a mean is a
    weight of 1 / rows).  Returns (loss, dlogits); dlogits may be given, also as the logits."""
    _on_device(logits=logits, top_ids=top_ids, top_logits=top_logits, weight=weight, dlogits=dlogits)
    d = _distill_params(logits, top_ids, top_logits, weight, temperature)
    loss = torch.empty(logits.shape[:-1], dtype=torch.float32, device=logits.device)
    dlogits, ld = _dlogits(logits, dlogits)
    _check(malt.load().malt_distill_forward_backward(d, loss.data_ptr(), 0, dlogits.data_ptr(), ld,
                                                     _stream(stream, loss, dlogits)), "malt_distill_forward_backward")
    return loss, dlogits
