"""What a language model does with a retrieval: ctypes binding of the calls under "reading" in
``include/logoskg.h``.  Argument checks and marshalling only; outputs and workspaces are torch tensors, nothing
synchronises.  With ``stream`` a call's work and its tensors belong to that stream (and the inputs must live until it is
through), else to torch's current one.

A small call's time is what happens here: a question's first token reads its 900 entities in 13 us of the GPU's time, and
the call took 19 us before tensors were asked for each property once and structures were packed (1.6 to 0.3 us)."""
from __future__ import annotations

import ctypes
import functools
import math
import struct

from .binding import _check, _load, _stream_handle, _torch

_P, _I32, _I64, _F = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float


class _Score(ctypes.Structure):
    _fields_ = [("scale", _F), ("cap", _F), ("bias", _P), ("buckets", _P), ("num_buckets", _I32), ("max_distance", _I32)]


class _Attention(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("device", _I32), ("dtype", _I32), ("num_docs", _I32), ("heads", _I32),
                ("kv_heads", _I32), ("dim", _I32), ("causal", _I32), ("num_rows", _I64), ("num_keys", _I64),
                ("q_off", _P), ("k_off", _P), ("q", _P), ("k", _P), ("v", _P), ("q_row", _I64), ("q_head", _I64),
                ("k_row", _I64), ("k_head", _I64), ("v_row", _I64), ("v_head", _I64), ("prefix", _P), ("q_pos", _P),
                ("k_pos", _P), ("score", _Score), ("out", _P), ("lse", _P), ("stream", _P)]


class _AttentionGrad(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("reserved", _I32), ("dout", _P), ("dq", _P), ("dk", _P), ("dv", _P),
                ("dbias", _P), ("workspace", _P), ("workspace_bytes", _I64)]


class _EntityRead(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("device", _I32), ("dtype", _I32), ("num_queries", _I32),
                ("tokens", _I32), ("heads", _I32), ("kv_heads", _I32), ("dim", _I32), ("num_entries", _I64),
                ("num_entities", _I64), ("off", _P), ("entity", _P), ("hop", _P), ("q_pos", _P), ("q", _P), ("keys", _P),
                ("values", _P), ("key_row", _I64), ("key_head", _I64), ("value_row", _I64), ("value_head", _I64),
                ("score", _Score), ("out", _P), ("lse", _P), ("workspace", _P), ("workspace_bytes", _I64), ("stream", _P)]


class _Logits(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("device", _I32), ("dtype", _I32), ("num_rows", _I32), ("vocab", _I64),
                ("row", _I64), ("logits", _P), ("out", _P), ("history_off", _P), ("history", _P), ("num_history", _I64),
                ("repetition", _P), ("presence", _P), ("frequency", _P), ("bias_off", _P), ("bias_id", _P),
                ("bias_value", _P), ("num_bias", _I64), ("mask", _P), ("stream", _P)]


def _packer(cls):
    """bytes of a structure from its fields' values in turn, those of a _Score inside as its six (NULL: 0)."""
    code = {ctypes.c_uint32: "I", _I32: "i", _I64: "q", _P: "Q", _F: "f", _Score: "ffQQii"}
    return struct.Struct("=" + "".join(code[kind] for _, kind in cls._fields_)).pack


_attention_of, _gradients_of, _entity_read_of, _logits_of = (_packer(c) for c in (_Attention, _AttentionGrad, _EntityRead, _Logits))
_TYPES = None  # torch type -> logoskg_dtype


def _dtype(dtype) -> int:
    global _TYPES
    if _TYPES is None:
        torch = _torch()
        _TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
    if dtype not in _TYPES:
        raise ValueError(f"{dtype} is not supported")
    return _TYPES[dtype]


def _on_stream(call):
    """``stream``: the call with that stream as torch's current one, so that its tensors are of that stream's memory."""
    @functools.wraps(call)
    def on(*args, stream=None, **kw):
        if stream is None:
            return call(*args, **kw)
        with _torch().cuda.stream(stream):
            return call(*args, **kw)
    return on


def _on_gpu(t, name) -> int:
    """The number of the tensor's GPU."""
    device = t.get_device()
    if device < 0:
        raise ValueError(f"{name} must be on the GPU (no CPU fallback)")
    return device


def _plain(t, name, dtype, device, shape=None) -> int:
    """The place of a contiguous tensor of that type on that GPU; 0 for None."""
    if t is None:
        return 0
    if t.dtype is not dtype or t.get_device() != device or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor on cuda:{device}")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name} has the shape {tuple(t.shape)}, not {shape}")
    return t.data_ptr()


def _rows(t, name, dtype, device):
    """Sizes and strides of the rows and heads of a [rows, heads, dim] tensor whose last axis is contiguous."""
    if t.dim() != 3 or t.dtype is not dtype or t.get_device() != device:
        raise ValueError(f"{name} must be a [rows, heads, dim] {dtype} tensor on cuda:{device}")
    n, heads, dim = t.shape
    row, head, one = t.stride()
    if one != 1 and dim > 1 and n and heads:
        raise ValueError(f"the last axis of {name} must be contiguous")
    return n, heads, dim, row if n > 1 else 0, head if heads > 1 else 0


def _score(scale, cap, bias, buckets, heads, dim, dtype, device):
    """The values of a _Score."""
    scale = dim ** -0.5 if scale is None and dim else scale or 0.0
    if bias is None:
        if buckets is not None:
            raise ValueError("buckets without a bias")
        return scale, cap or 0.0, 0, 0, 0, 0
    if buckets is None or buckets.dim() != 1 or buckets.numel() % 2 != 1:
        raise ValueError("a bias needs buckets, one per distance -M .. M")
    if bias.dim() != 2 or bias.shape[0] != heads or bias.shape[1] < 1:
        raise ValueError("bias must be [heads, buckets], with a bucket at least")
    return (scale, cap or 0.0, _plain(bias, "bias", dtype, device), _plain(buckets, "buckets", _torch().int32, device),
            bias.shape[1], buckets.numel() // 2)


def _workspace(nbytes, like):
    if nbytes <= 0:
        if nbytes < 0:
            _check(1)  # (the library has said why)
        return None
    return like.new_empty(nbytes, dtype=_torch().uint8)


def distance_buckets(num_buckets: int, max_distance: int, both_sides: bool = True, device="cuda"):
    """int32[2 M + 1]: a bucket for every distance -M .. M (M = max_distance; what is farther counts as M).

    The near half of the buckets hold one distance each, the rest share the others by their logarithm.
    ``both_sides``: half of the buckets for either sign; else distances above 0 share bucket 0 with 0."""
    side = num_buckets // 2 if both_sides else num_buckets
    near = max(side // 2, 1)
    if side < 1 or max_distance < near:
        raise ValueError("too few buckets, or max_distance below the buckets of single distances")
    got = []
    for d in range(-max_distance, max_distance + 1):
        n = abs(d) if both_sides else max(-d, 0)
        if n >= near:
            far = math.log(n / near) / math.log(max_distance / near) if max_distance > near else 1.0
            n = min(near + int(far * (side - near)), side - 1)
        got.append(n + (side if both_sides and d > 0 else 0))
    torch = _torch()
    return torch.tensor(got, dtype=torch.int32, device=device)


def _attention(q, k, v, q_off, k_off, scale, cap, causal, prefix, bias, buckets, q_pos, k_pos, out, lse, stream):
    """An _Attention, packed."""
    torch = _torch()
    dtype, device = q.dtype, _on_gpu(q, "q")
    n, heads, dim, q_row, q_head = _rows(q, "q", dtype, device)
    m, kv_heads, k_dim, k_row, k_head = _rows(k, "k", dtype, device)
    v_row, v_head = _rows(v, "v", dtype, device)[3:]
    if v.shape != k.shape or k_dim != dim:
        raise ValueError("k and v must have one shape, and q's head size")
    docs = q_off.numel() - 1
    if k_off.numel() - 1 != docs or docs < 0:
        raise ValueError("q_off and k_off must have one entry per document and one more")
    if prefix is not None and not causal:
        raise ValueError("a prefix is part of the causal mask")
    return _attention_of(
            216, device, _dtype(dtype), docs, heads, kv_heads, dim, 1 if causal else 0, n, m,
            _plain(q_off, "q_off", torch.int64, device), _plain(k_off, "k_off", torch.int64, device), q.data_ptr(), k.data_ptr(),
            v.data_ptr(), q_row, q_head, k_row, k_head, v_row, v_head, _plain(prefix, "prefix", torch.int32, device, (docs,)),
            _plain(q_pos, "q_pos", torch.int32, device, (n,)), _plain(k_pos, "k_pos", torch.int32, device, (m,)),
            *_score(scale, cap, bias, buckets, heads, dim, dtype, device), out.data_ptr(), lse.data_ptr(), _stream_handle(stream, device))


def _new(t):
    return _torch().empty_like(t) if t.is_contiguous() else t.new_empty(t.shape)


@functools.lru_cache(None)
def _differentiable():
    torch = _torch()

    class Attend(torch.autograd.Function):
        """``attend`` for inputs that require gradients."""

        @staticmethod
        def forward(ctx, q, k, v, bias, q_off, k_off, kw):
            out, lse = attend(q, k, v, q_off, k_off, bias=bias, **kw)
            ctx.set_materialize_grads(False)
            ctx.save_for_backward(q, k, v, bias, out, lse, q_off, k_off)
            ctx.kw = kw
            return out, lse

        @staticmethod
        @torch.autograd.function.once_differentiable
        def backward(ctx, dout, dlse):
            if dlse is not None:
                raise RuntimeError("attend: lse has no gradient (parts that are joined by it cannot be trained)")
            if dout is None:
                return (None,) * 7
            q, k, v, bias, out, lse, q_off, k_off = ctx.saved_tensors
            return (*attend_backward(dout.contiguous(), q, k, v, out, lse, q_off, k_off, bias=bias, **ctx.kw), None, None, None)

    return Attend


@_on_stream
def attend(q, k, v, q_off, k_off, *, scale=None, cap=0.0, causal=False, prefix=None, bias=None, buckets=None, q_pos=None,
           k_pos=None):
    """``logoskg_attend``: attention of a ragged batch, as (out [rows, heads, dim], lse float32 [rows, heads]).

    ``q`` [rows, heads, dim], ``k`` and ``v`` [keys, kv_heads, dim] in bfloat16 or float16, documents one behind the
    other at ``q_off`` / ``k_off`` (int64, on the device); rows that none holds get zeros and -inf.  ``causal``: row i of R sees the keys up to i + K - R, and
    the document's first ``prefix`` (int32, one per document) besides; else every row sees all keys.  ``cap``: scores
    become cap tanh(score / cap).  ``bias`` [heads, buckets] is learned, ``buckets`` (``distance_buckets``) says which
    column the distance ``k_pos - q_pos`` reads (positions: int32, by default the places, aligned at the end).

    Where ``q``, ``k``, ``v`` or ``bias`` requires a gradient, ``out`` has one by ``attend_backward``; ``lse`` has none, and
    asking for it raises."""
    if (q.requires_grad or k.requires_grad or v.requires_grad or bias is not None and bias.requires_grad) and _torch().is_grad_enabled():
        kw = dict(scale=scale, cap=cap, causal=causal, prefix=prefix, buckets=buckets, q_pos=q_pos, k_pos=k_pos)
        return _differentiable().apply(q, k, v, bias, q_off, k_off, kw)
    out, lse = _new(q), q.new_empty(q.shape[:2], dtype=_torch().float32)
    _check(_load().logoskg_attend(_attention(q, k, v, q_off, k_off, scale, cap, causal, prefix, bias, buckets, q_pos, k_pos, out, lse, None)))
    return out, lse


@_on_stream
def attend_backward(dout, q, k, v, out, lse, q_off, k_off, *, scale=None, cap=0.0, causal=False, prefix=None, bias=None,
                    buckets=None, q_pos=None, k_pos=None):
    """``logoskg_attend_backward``: gradients (dq, dk, dv, dbias or None) for ``dout``, the gradient of ``attend``'s
    ``out``; the other arguments are those of that call and what it returned.  The same inputs give the same bits."""
    torch = _torch()
    device = _on_gpu(q, "q")
    dout_at = _plain(dout, "dout", q.dtype, device, q.shape)
    _plain(out, "out", q.dtype, device, q.shape)
    _plain(lse, "lse", torch.float32, device, q.shape[:2])
    a = _attention(q, k, v, q_off, k_off, scale, cap, causal, prefix, bias, buckets, q_pos, k_pos, out, lse, None)
    dq, dk, dv = _new(q), _new(k), _new(v)
    dbias = None if bias is None else torch.empty_like(bias)
    lib = _load()
    w = _workspace(lib.logoskg_attend_backward_bytes(a), q)
    g = _gradients_of(64, 0, dout_at, dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), 0 if dbias is None else dbias.data_ptr(),
                      *((0, 0) if w is None else (w.data_ptr(), w.numel())))
    _check(lib.logoskg_attend_backward(a, g))
    return dq, dk, dv, dbias


@_on_stream
def read_entities(q, keys, values, off, entity=None, *, scale=None, cap=0.0, bias=None, buckets=None, hop=None, q_pos=None):
    """``logoskg_read_entities``: the tokens of every query attend to its entity list, as {"out": like q, "lse":
    float32 [queries, tokens, heads]} (with its lse, the answer can be joined with attention over the text).  A serving call: it
    has no gradient.

    ``q`` [queries, tokens, heads, dim]; ``keys`` / ``values`` [entities, kv_heads, dim] by entity; ``off`` (int64),
    ``entity`` (int32) and ``hop`` (uint8) as ``Result.offsets`` and ``Result.fetch`` give them, on the device.  An entity
    stands at its hop, a token at ``q_pos`` (int32 per query, 0 by default).  Without ``entity`` entry i reads row i."""
    torch = _torch()
    if q.dim() != 4 or not q.is_contiguous():
        raise ValueError("q must be a contiguous [queries, tokens, heads, dim] tensor")
    dtype, device = q.dtype, _on_gpu(q, "q")
    n, tokens, heads, dim = q.shape
    rows, kv_heads, k_dim, k_row, k_head = _rows(keys, "keys", dtype, device)
    v_row, v_head = _rows(values, "values", dtype, device)[3:]
    if values.shape != keys.shape or k_dim != dim:
        raise ValueError("keys and values must have one shape, and q's head size")
    entries = rows if entity is None else entity.numel()
    head = (208, device, _dtype(dtype), n, tokens, heads, kv_heads, dim, entries, rows, _plain(off, "off", torch.int64, device, (n + 1,)),
            _plain(entity, "entity", torch.int32, device, (entries,)), _plain(hop, "hop", torch.uint8, device, (entries,)),
            _plain(q_pos, "q_pos", torch.int32, device, (n,)), q.data_ptr(), keys.data_ptr(), values.data_ptr(), k_row, k_head,
            v_row, v_head, *_score(scale, cap, bias, buckets, heads, dim, dtype, device))
    out, lse = torch.empty_like(q), q.new_empty((n, tokens, heads), dtype=torch.float32)
    head += (out.data_ptr(), lse.data_ptr())
    lib = _load()
    w = _workspace(lib.logoskg_read_entities_bytes(_entity_read_of(*head, 0, 0, 0)), q)
    _check(lib.logoskg_read_entities(_entity_read_of(*head, *((0, 0) if w is None else (w.data_ptr(), w.numel())),
                                                     _stream_handle(None, device))))
    return {"out": out, "lse": lse}


@_on_stream
def entity_mask(off, ids, num_ids: int, *, out=None):
    """``logoskg_entity_mask``: int64[queries, ceil(num_ids / 64)] words, bit i % 64 of word i / 64 set for the ids of a
    query's list (``off`` int64, ``ids`` int32 on the device, any order): the layout of ``Graph.khop``'s ``rel_mask``."""
    torch = _torch()
    device = _on_gpu(ids, "ids")
    off_at, ids_at = _plain(off, "off", torch.int64, device), _plain(ids, "ids", torch.int32, device)
    queries = off.numel() - 1
    if queries < 0:
        raise ValueError("off must have one entry per query and one more")
    shape = (queries, (num_ids + 63) // 64)
    if out is None:
        out = off.new_empty(shape)
    _check(_load().logoskg_entity_mask(device, off_at, ids_at, ids.numel(), queries, num_ids,
                                       _plain(out, "out", torch.int64, device, shape), _stream_handle(None, device)))
    return out


@_on_stream
def constrain_logits(logits, *, history=None, history_off=None, repetition=None, presence=None, frequency=None,
                     bias_off=None, bias_id=None, bias_value=None, mask=None, out=None):
    """``logoskg_constrain_logits``: a step's logits [rows, vocab] (bfloat16, float16 or float32) with the ids of each
    row's ``history`` penalised (``repetition`` divides or multiplies, ``presence`` and count times ``frequency`` are taken
    off; float32 per row), biases added, and every id whose bit of ``mask`` (``entity_mask``'s layout) is 0 at -infinity.
    Lists are ragged: ``history`` int32 at ``history_off``, ``bias_id`` int32 and ``bias_value`` float32 at ``bias_off``.
    ``out`` may be ``logits``.  A serving call: it has no gradient."""
    torch = _torch()
    if logits.dim() != 2:
        raise ValueError("logits must be [rows, vocab] with contiguous rows")
    (rows, vocab), (row, one) = logits.shape, logits.stride()
    if one != 1 and rows and vocab > 1:
        raise ValueError("logits must be [rows, vocab] with contiguous rows")
    device = _on_gpu(logits, "logits")
    if (history is None) != (history_off is None) or (bias_id is None) != (bias_off is None) or (bias_id is None) != (bias_value is None):
        raise ValueError("history comes with history_off, and bias_id with bias_off and bias_value")
    if history is None and not (repetition is None and presence is None and frequency is None):
        raise ValueError("penalties without a history")
    int32, int64, float32, per_row = torch.int32, torch.int64, torch.float32, (rows,)
    head = (144, device, _dtype(logits.dtype), rows, vocab, row if rows > 1 else vocab, logits.data_ptr())
    tail = (_plain(history_off, "history_off", int64, device, (rows + 1,)), _plain(history, "history", int32, device),
            0 if history is None else history.numel(), _plain(repetition, "repetition", float32, device, per_row),
            _plain(presence, "presence", float32, device, per_row), _plain(frequency, "frequency", float32, device, per_row),
            _plain(bias_off, "bias_off", int64, device, (rows + 1,)), _plain(bias_id, "bias_id", int32, device),
            _plain(bias_value, "bias_value", float32, device, None if bias_id is None else bias_id.shape),
            0 if bias_id is None else bias_id.numel(), _plain(mask, "mask", int64, device, (rows, (vocab + 63) // 64)))
    if out is None:
        out = torch.empty_like(logits) if logits.is_contiguous() else torch.empty_strided((rows, vocab), (row, one), dtype=logits.dtype, device=logits.device)
    elif out.shape != logits.shape or out.dtype is not logits.dtype or out.get_device() != device or out.stride() != (row, one):
        raise ValueError("out must be laid out as logits")
    _check(_load().logoskg_constrain_logits(_logits_of(*head, out.data_ptr(), *tail, _stream_handle(None, device))))
    return out
