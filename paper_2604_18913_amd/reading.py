"""What a language model does with a retrieval: ctypes binding of the calls under "reading" in
``include/logoskg.h``.  Argument checks and marshalling only; outputs and workspaces are torch
tensors of the current stream's allocator, nothing synchronises."""
from __future__ import annotations

import ctypes
import math

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


_TYPES = None  # torch type -> logoskg_dtype


def _dtype(t) -> int:
    global _TYPES
    if _TYPES is None:
        torch = _torch()
        _TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
    if t.dtype not in _TYPES:
        raise ValueError(f"{t.dtype} is not supported")
    return _TYPES[t.dtype]


def _ptr(t):
    return None if t is None else t.data_ptr()


def _plain(t, name, dtype, device, shape=None):
    """A contiguous tensor of that type on the device, or None."""
    if t is None:
        return None
    if t.dtype != dtype or t.device != device or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor on {device}")
    if shape is not None and tuple(t.shape) != shape:
        raise ValueError(f"{name} has the shape {tuple(t.shape)}, not {shape}")
    return t


def _rows(t, name, dtype, device):
    """A [rows, heads, dim] tensor whose last axis is contiguous; the strides of the others are free."""
    if t.dim() != 3 or t.dtype != dtype or t.device != device:
        raise ValueError(f"{name} must be a [rows, heads, dim] {dtype} tensor on {device}")
    if t.numel() and t.shape[2] > 1 and t.stride(2) != 1:
        raise ValueError(f"the last axis of {name} must be contiguous")
    return t


def _score(scale, cap, bias, buckets, heads, dim, dtype, device):
    if bias is None:
        if buckets is not None:
            raise ValueError("buckets without a bias")
        return _Score(1.0 / math.sqrt(dim) if scale is None else scale, cap or 0.0, None, None, 0, 0)
    if buckets is None or buckets.dim() != 1 or buckets.numel() % 2 != 1:
        raise ValueError("a bias needs buckets, one per distance -M .. M")
    torch = _torch()
    if bias.dim() != 2 or bias.shape[0] != heads:
        raise ValueError("bias must be [heads, buckets]")
    _plain(bias, "bias", dtype, device)
    _plain(buckets, "buckets", torch.int32, device)
    return _Score(1.0 / math.sqrt(dim) if scale is None else scale, cap or 0.0, bias.data_ptr(), buckets.data_ptr(),
                  bias.shape[1], buckets.numel() // 2)


def _on_gpu(t, name):
    if t.device.type != "cuda":
        raise ValueError(f"{name} must be on the GPU (no CPU fallback)")
    return t.device


def _workspace(nbytes, device, stream):
    if nbytes < 0:
        _check(1)  # (the library has said why)
    if nbytes == 0:
        return None
    torch = _torch()
    w = torch.empty(nbytes, dtype=torch.uint8, device=device)
    if stream is not None:
        w.record_stream(stream)
    return w


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
    torch = _torch()
    dtype, device = q.dtype, _on_gpu(q, "q")
    for t, name in ((q, "q"), (k, "k"), (v, "v")):
        _rows(t, name, dtype, device)
    n, heads, dim = q.shape
    m, kv_heads = k.shape[:2]
    if v.shape != k.shape or k.shape[2] != dim:
        raise ValueError("k and v must have one shape, and q's head size")
    docs = q_off.numel() - 1
    if k_off.numel() - 1 != docs or docs < 0:
        raise ValueError("q_off and k_off must have one entry per document and one more")
    _plain(q_off, "q_off", torch.int64, device)
    _plain(k_off, "k_off", torch.int64, device)
    _plain(prefix, "prefix", torch.int32, device, (docs,))
    _plain(q_pos, "q_pos", torch.int32, device, (n,))
    _plain(k_pos, "k_pos", torch.int32, device, (m,))
    if prefix is not None and not causal:
        raise ValueError("a prefix is part of the causal mask")
    s = _score(scale, cap, bias, buckets, heads, dim, dtype, device)
    return _Attention(ctypes.sizeof(_Attention), device.index or 0, _dtype(q), docs, heads, kv_heads, dim, 1 if causal else 0, n, m,
                      q_off.data_ptr(), k_off.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(), q.stride(0), q.stride(1),
                      k.stride(0), k.stride(1), v.stride(0), v.stride(1), _ptr(prefix), _ptr(q_pos), _ptr(k_pos), s,
                      out.data_ptr(), lse.data_ptr(), _stream_handle(stream))


def attend(q, k, v, q_off, k_off, *, scale=None, cap=0.0, causal=False, prefix=None, bias=None, buckets=None, q_pos=None,
           k_pos=None, stream=None):
    """``logoskg_attend``: attention of a ragged batch, as (out [rows, heads, dim], lse float32 [rows, heads]).

    ``q`` [rows, heads, dim], ``k`` and ``v`` [keys, kv_heads, dim] in bfloat16 or float16, documents one behind the
    other at ``q_off`` / ``k_off`` (int64, on the device).  ``causal``: row i of R sees the keys up to i + K - R, and
    the document's first ``prefix`` (int32, one per document) besides; else every row sees all keys.  ``cap``: scores
    become cap tanh(score / cap).  ``bias`` [heads, buckets] is learned, ``buckets`` (``distance_buckets``) says which
    column the distance ``k_pos - q_pos`` reads (positions: int32, by default the places, aligned at the end)."""
    torch = _torch()
    out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    lse = torch.empty(q.shape[:2], dtype=torch.float32, device=q.device)
    a = _attention(q, k, v, q_off, k_off, scale, cap, causal, prefix, bias, buckets, q_pos, k_pos, out, lse, stream)
    _check(_load().logoskg_attend(ctypes.addressof(a)))
    return out, lse


def attend_backward(dout, q, k, v, out, lse, q_off, k_off, *, scale=None, cap=0.0, causal=False, prefix=None, bias=None,
                    buckets=None, q_pos=None, k_pos=None, stream=None):
    """``logoskg_attend_backward``: gradients (dq, dk, dv, dbias or None) for ``dout``, the gradient of ``attend``'s
    ``out``; the other arguments are those of that call and what it returned.  The same inputs give the same bits."""
    torch = _torch()
    _plain(dout, "dout", q.dtype, q.device, tuple(q.shape))
    _plain(out, "out", q.dtype, q.device, tuple(q.shape))
    _plain(lse, "lse", torch.float32, q.device, tuple(q.shape[:2]))
    a = _attention(q, k, v, q_off, k_off, scale, cap, causal, prefix, bias, buckets, q_pos, k_pos, out, lse, stream)
    dq, dk, dv = (torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in (q, k, v))
    dbias = None if bias is None else torch.empty_like(bias)
    lib = _load()
    w = _workspace(lib.logoskg_attend_backward_bytes(ctypes.addressof(a)), q.device, stream)
    g = _AttentionGrad(ctypes.sizeof(_AttentionGrad), 0, dout.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(),
                       _ptr(dbias), _ptr(w), 0 if w is None else w.numel())
    _check(lib.logoskg_attend_backward(ctypes.addressof(a), ctypes.addressof(g)))
    return dq, dk, dv, dbias


def read_entities(q, keys, values, off, entity=None, *, scale=None, cap=0.0, bias=None, buckets=None, hop=None, q_pos=None,
                  stream=None):
    """``logoskg_read_entities``: the tokens of every query attend to its entity list, as {"out": like q, "lse":
    float32 [queries, tokens, heads]} (with its lse, the answer can be joined with attention over the text).

    ``q`` [queries, tokens, heads, dim]; ``keys`` / ``values`` [entities, kv_heads, dim] by entity; ``off`` (int64),
    ``entity`` (int32) and ``hop`` (uint8) as ``Result.offsets`` and ``Result.fetch`` give them, on the device.  An entity
    stands at its hop, a token at ``q_pos`` (int32 per query, 0 by default).  Without ``entity`` entry i reads row i."""
    torch = _torch()
    if q.dim() != 4 or not q.is_contiguous():
        raise ValueError("q must be a contiguous [queries, tokens, heads, dim] tensor")
    _on_gpu(q, "q")
    n, tokens, heads, dim = q.shape
    _rows(keys, "keys", q.dtype, q.device)
    _rows(values, "values", q.dtype, q.device)
    if values.shape != keys.shape or keys.shape[2] != dim:
        raise ValueError("keys and values must have one shape, and q's head size")
    entries = keys.shape[0] if entity is None else entity.numel()
    _plain(off, "off", torch.int64, q.device, (n + 1,))
    _plain(entity, "entity", torch.int32, q.device, (entries,))
    _plain(hop, "hop", torch.uint8, q.device, (entries,))
    _plain(q_pos, "q_pos", torch.int32, q.device, (n,))
    s = _score(scale, cap, bias, buckets, heads, dim, q.dtype, q.device)
    out = torch.empty_like(q)
    lse = torch.empty((n, tokens, heads), dtype=torch.float32, device=q.device)
    r = _EntityRead(ctypes.sizeof(_EntityRead), q.device.index or 0, _dtype(q), n, tokens, heads, keys.shape[1], dim, entries,
                    keys.shape[0], off.data_ptr(), _ptr(entity), _ptr(hop), _ptr(q_pos), q.data_ptr(), keys.data_ptr(),
                    values.data_ptr(), keys.stride(0), keys.stride(1), values.stride(0), values.stride(1), s, out.data_ptr(),
                    lse.data_ptr(), None, 0, _stream_handle(stream))
    lib = _load()
    w = _workspace(lib.logoskg_read_entities_bytes(ctypes.addressof(r)), q.device, stream)
    if w is not None:
        r.workspace, r.workspace_bytes = w.data_ptr(), w.numel()
    _check(lib.logoskg_read_entities(ctypes.addressof(r)))
    return {"out": out, "lse": lse}


def entity_mask(off, ids, num_ids: int, *, out=None, stream=None):
    """``logoskg_entity_mask``: int64[queries, ceil(num_ids / 64)] words, bit i % 64 of word i / 64 set for the ids of a
    query's list (``off`` int64, ``ids`` int32 on the device, any order): the layout of ``Graph.khop``'s ``rel_mask``."""
    torch = _torch()
    _plain(ids, "ids", torch.int32, _on_gpu(ids, "ids"))
    _plain(off, "off", torch.int64, ids.device)
    shape = (off.numel() - 1, (num_ids + 63) // 64)
    if out is None:
        out = torch.empty(shape, dtype=torch.int64, device=ids.device)
    _plain(out, "out", torch.int64, ids.device, shape)
    _check(_load().logoskg_entity_mask(ids.device.index or 0, off.data_ptr(), ids.data_ptr(), ids.numel(), shape[0], num_ids,
                                       out.data_ptr(), _stream_handle(stream)))
    return out


def constrain_logits(logits, *, history=None, history_off=None, repetition=None, presence=None, frequency=None,
                     bias_off=None, bias_id=None, bias_value=None, mask=None, out=None, stream=None):
    """``logoskg_constrain_logits``: a step's logits [rows, vocab] (bfloat16, float16 or float32) with the ids of each
    row's ``history`` penalised (``repetition`` divides or multiplies, ``presence`` and count times ``frequency`` are taken
    off; float32 per row), biases added, and every id whose bit of ``mask`` (``entity_mask``'s layout) is 0 at -infinity.
    Lists are ragged: ``history`` int32 at ``history_off``, ``bias_id`` int32 and ``bias_value`` float32 at ``bias_off``.
    ``out`` may be ``logits``."""
    torch = _torch()
    if logits.dim() != 2 or (logits.numel() and logits.stride(1) != 1):
        raise ValueError("logits must be [rows, vocab] with contiguous rows")
    rows, vocab = logits.shape
    device = _on_gpu(logits, "logits")
    if (history is None) != (history_off is None) or (bias_id is None) != (bias_off is None) or (bias_id is None) != (bias_value is None):
        raise ValueError("history comes with history_off, and bias_id with bias_off and bias_value")
    if history is None and not (repetition is None and presence is None and frequency is None):
        raise ValueError("penalties without a history")
    for t, name in ((history_off, "history_off"), (bias_off, "bias_off")):
        _plain(t, name, torch.int64, device, (rows + 1,))
    for t, name in ((repetition, "repetition"), (presence, "presence"), (frequency, "frequency")):
        _plain(t, name, torch.float32, device, (rows,))
    _plain(history, "history", torch.int32, device)
    _plain(bias_id, "bias_id", torch.int32, device)
    _plain(bias_value, "bias_value", torch.float32, device, None if bias_id is None else tuple(bias_id.shape))
    _plain(mask, "mask", torch.int64, device, (rows, (vocab + 63) // 64))
    if out is None:
        out = torch.empty_strided(logits.shape, logits.stride(), dtype=logits.dtype, device=device)
    elif out.shape != logits.shape or out.dtype != logits.dtype or out.device != device or out.stride() != logits.stride():
        raise ValueError("out must be laid out as logits")
    a = _Logits(ctypes.sizeof(_Logits), device.index or 0, _dtype(logits), rows, vocab, logits.stride(0) if rows > 1 else vocab,
                logits.data_ptr(), out.data_ptr(), _ptr(history_off), _ptr(history), 0 if history is None else history.numel(),
                _ptr(repetition), _ptr(presence), _ptr(frequency), _ptr(bias_off), _ptr(bias_id), _ptr(bias_value),
                0 if bias_id is None else bias_id.numel(), _ptr(mask), _stream_handle(stream))
    _check(_load().logoskg_constrain_logits(ctypes.addressof(a)))
    return out
