"""Tables of keys and values by entity in 4 bits: ctypes binding of the calls under "tables in 4 bits" in ``include/logoskg.h``, in
the manner of ``reading``.  A 3,000,000-entity table of 8 key heads of 128 takes 3.8 GB instead of the 12.3 of 16 bits."""
from __future__ import annotations

import ctypes
import functools

from .binding import _check, _load, _stream_handle, _torch
from .reading import _apart, _dtype, _entity_read_of, _I32, _I64, _last_of, _on_gpu, _on_stream, _P, _packer, _plain, _rows, _score, _workspace


class _Pack(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("device", _I32), ("dtype", _I32), ("kv_heads", _I32), ("dim", _I32), ("reserved", _I32),
                ("num_rows", _I64), ("keys", _P), ("values", _P), ("key_row", _I64), ("key_head", _I64), ("value_row", _I64),
                ("value_head", _I64), ("packed", _P), ("packed_row", _I64), ("stream", _P)]


_pack_of = _packer(_Pack)


@functools.lru_cache(None)
def packed_row_bytes(kv_heads: int, dim: int) -> int:
    """``logoskg_packed_row_bytes``: the bytes of a packed row, 40 for every head and 32 elements of ``dim``."""
    n = _load().logoskg_packed_row_bytes(kv_heads, dim)
    if n == 0:
        raise ValueError("dim must be a multiple of 8 up to 128, and kv_heads positive")
    return n


def _packed_rows(t, name, nbytes, device):
    """Rows and their stride of a [rows, bytes] uint8 tensor."""
    if t.dim() != 2 or t.dtype is not _torch().uint8 or t.get_device() != device or t.shape[1] != nbytes:
        raise ValueError(f"{name} must be a [rows, {nbytes}] uint8 tensor on cuda:{device}")
    n, (row, one) = t.shape[0], t.stride()
    if one != 1 and n:
        raise ValueError(f"the last axis of {name} must be contiguous")
    return n, row if n > 1 else nbytes


@_on_stream
def pack_entities(keys, values, *, out=None):
    """``logoskg_pack_entities``: ``keys`` and ``values`` [entities, kv_heads, dim] (bfloat16, float16 or float32) in 4 bits, as
    uint8 [entities, packed_row_bytes(kv_heads, dim)] for ``read_packed``.  ``out`` may be rows of a larger table:
    ``pack_entities(k, v, out=table[a:b])``; single rows are replaced as any tensor's, ``table[ids] = pack_entities(k, v)``.

    Groups of 32 elements of a head have a scale and a base in bfloat16, a fifteenth of the group's range being a step; the layout and
    what it loses stand in ``include/logoskg.h`` (a group that stands far from 0 against its range loses most).  A group with an infinity or NaN becomes NaN.  There is no gradient."""
    torch = _torch()
    dtype, device = keys.dtype, _on_gpu(keys, "keys")
    n, heads, dim, k_row, k_head = _rows(keys, "keys", dtype, device)
    v_row, v_head = _rows(values, "values", dtype, device)[3:]
    if values.shape != keys.shape:
        raise ValueError("keys and values must have one shape")
    nbytes = packed_row_bytes(heads, dim)
    if out is None:
        out = keys.new_empty((n, nbytes), dtype=torch.uint8)
    else:
        _apart(out, "out", keys, values)
    rows, row = _packed_rows(out, "out", nbytes, device)
    if rows != n:
        raise ValueError(f"out has {rows} rows, not {n}")
    _check(_load().logoskg_pack_entities(_pack_of(104, device, _dtype(dtype), heads, dim, 0, n, keys.data_ptr(), values.data_ptr(), k_row,
                                                  k_head, v_row, v_head, out.data_ptr(), row, _stream_handle(None, device))))
    return out


@_on_stream
def unpack_entities(packed, kv_heads: int, dim: int, *, dtype):
    """``logoskg_unpack_entities``: the keys and values [rows, kv_heads, dim] that packed rows stand for, in ``dtype``."""
    torch = _torch()
    device = _on_gpu(packed, "packed")
    n, row = _packed_rows(packed, "packed", packed_row_bytes(kv_heads, dim), device)
    keys = packed.new_empty((n, kv_heads, dim), dtype=dtype)
    values = torch.empty_like(keys)
    _check(_load().logoskg_unpack_entities(_pack_of(104, device, _dtype(dtype), kv_heads, dim, 0, n, keys.data_ptr(), values.data_ptr(),
                                                    kv_heads * dim, dim, kv_heads * dim, dim, packed.data_ptr(), row,
                                                    _stream_handle(None, device))))
    return keys, values


@_on_stream
def read_packed(q, packed, off, entity=None, *, kv_heads, scale=None, cap=0.0, bias=None, buckets=None, hop=None, q_pos=None):
    """``logoskg_read_packed``: ``read_entities`` of a table by ``pack_entities``, as {"out": like q, "lse": float32 [queries, tokens,
    heads]}.  The other arguments are ``read_entities``'s; ``q`` (bfloat16 or float16) decides the type of ``out``, whatever
    type the table was packed from.  A serving call: it has no gradient."""
    torch = _torch()
    if q.dim() != 4 or not q.is_contiguous():
        raise ValueError("q must be a contiguous [queries, tokens, heads, dim] tensor")
    dtype, device = q.dtype, _on_gpu(q, "q")
    n, tokens, heads, dim = q.shape
    rows, row = _packed_rows(packed, "packed", packed_row_bytes(kv_heads, dim), device)
    entries = rows if entity is None else entity.numel()
    head = (208, device, _dtype(dtype), n, tokens, heads, kv_heads, dim, entries, rows, _plain(off, "off", torch.int64, device, (n + 1,)),
            _plain(entity, "entity", torch.int32, device, (entries,)), _plain(hop, "hop", torch.uint8, device, (entries,)),
            _plain(q_pos, "q_pos", torch.int32, device, (n,)), q.data_ptr(), packed.data_ptr(), 0, row, 0, 0, 0,
            *_score(scale, cap, bias, buckets, heads, dim, dtype, device))
    out, lse = torch.empty_like(q), q.new_empty((n, tokens, heads), dtype=torch.float32)
    head += (out.data_ptr(), lse.data_ptr())
    lib = _load()
    call = _entity_read_of(*head, 0, 0, 0)
    w = _workspace(lib.logoskg_read_packed_bytes(call), q)
    _check(lib.logoskg_read_packed(call[:-24] + _last_of(*((0, 0) if w is None else (w.data_ptr(), w.numel())), _stream_handle(None, device))))
    return {"out": out, "lse": lse}
