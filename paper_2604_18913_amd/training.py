"""Around the reading of a retrieval in training: rows of an entity table and their gradient, the loss of sampled answers, the
end of a step.  ctypes binding of the calls under "around the reading" in ``include/logoskg.h``, in the manner of ``reading``:
outputs and workspaces are torch tensors, nothing synchronises, and with ``stream`` a call's work and tensors belong to that
stream."""
from __future__ import annotations

import ctypes
import functools
import struct

from .binding import _check, _load, _stream_handle, _torch
from .reading import _apart, _dtype, _F, _has_tangent, _I32, _I64, _last_of, _on_gpu, _on_stream, _P, _packer, _plain, _workspace

_U32 = ctypes.c_uint32


class _Embedding(ctypes.Structure):
    _fields_ = [("struct_size", _U32), ("device", _I32), ("dtype", _I32), ("scale", _F), ("num_ids", _I64), ("num_entities", _I64),
                ("dim", _I64), ("row", _I64), ("ids", _P), ("table", _P), ("out", _P), ("stream", _P)]


class _EmbeddingGrad(ctypes.Structure):
    _fields_ = [("struct_size", _U32), ("device", _I32), ("dtype", _I32), ("table_dtype", _I32), ("scale", _F), ("accumulate", _I32),
                ("num_ids", _I64), ("num_entities", _I64), ("dim", _I64), ("row", _I64), ("ids", _P), ("dout", _P), ("dtable", _P),
                ("workspace", _P), ("workspace_bytes", _I64), ("stream", _P)]


class _Policy(ctypes.Structure):
    _fields_ = [("struct_size", _U32), ("device", _I32), ("dtype", _I32), ("num_rows", _I32), ("vocab", _I64), ("row", _I64),
                ("logits", _P), ("target", _P), ("mask", _P), ("mask_row", _P), ("num_masks", _I64), ("scale", _F), ("kl", _F),
                ("clip_low", _F), ("clip_high", _F), ("advantage", _P), ("old", _P), ("ref", _P), ("weight", _P), ("logp", _P),
                ("lse", _P), ("loss", _P), ("dlogits", _P), ("dloss", _P), ("stream", _P)]


class _Gradient(ctypes.Structure):
    _fields_ = [("grad", _P), ("out", _P), ("n", _I64), ("dtype", _I32), ("out_dtype", _I32)]


_embedding_of, _embedding_grad_of, _policy_of = (_packer(c) for c in (_Embedding, _EmbeddingGrad, _Policy))


# ---------------------------------------------------------------- rows of a table
def _table(t, name, dtype=None, device=None):
    """Sizes and row stride of a [entities, dim] tensor whose last axis is contiguous."""
    if t.dim() != 2 or (dtype is not None and t.dtype is not dtype) or (device is not None and t.get_device() != device):
        raise ValueError(f"{name} must be an [entities, dim] tensor" + (f" in {dtype} on cuda:{device}" if dtype is not None else ""))
    (n, dim), (row, one) = t.shape, t.stride()
    if one != 1 and n and dim > 1:
        raise ValueError(f"the last axis of {name} must be contiguous")
    return n, dim, row if n > 1 else dim


@functools.lru_cache(None)
def _differentiable_embedding():
    torch = _torch()

    class Embed(torch.autograd.Function):
        """``embed_entities`` of a table that requires a gradient."""

        @staticmethod
        def forward(ctx, table, ids, scale):
            ctx.save_for_backward(ids)
            ctx.num_entities, ctx.scale = table.shape[0], scale
            return embed_entities(table, ids, scale=scale)

        @staticmethod
        @torch.autograd.function.once_differentiable
        def backward(ctx, dout):
            ids, = ctx.saved_tensors
            return embed_entities_backward(dout.contiguous(), ids, ctx.num_entities, scale=ctx.scale), None, None

    return Embed


@_on_stream
def embed_entities(table, ids, *, scale=1.0):
    """``logoskg_embed_entities``: rows of ``table`` [entities, dim] (bfloat16, float16 or float32) by ``ids`` (int32 of any shape,
    as ``Result.fetch`` gives them) times ``scale``, as [*ids.shape, dim] in the table's type.  Ids outside the table pad: their rows are
    zeros.  Where ``table`` requires a gradient, the result has one by ``embed_entities_backward``."""
    torch = _torch()
    if table.requires_grad and torch.is_grad_enabled() or _has_tangent(table):
        return _differentiable_embedding().apply(table, ids, scale)
    device = _on_gpu(table, "table")
    entities, dim, row = _table(table, "table")
    at = _plain(ids, "ids", torch.int32, device)
    out = table.new_empty((*ids.shape, dim))
    _check(_load().logoskg_embed_entities(_embedding_of(80, device, _dtype(table.dtype), scale, ids.numel(), entities, dim, row, at,
                                                        table.data_ptr(), out.data_ptr(), _stream_handle(None, device))))
    return out


@_on_stream
def embed_entities_backward(dout, ids, num_entities, *, scale=1.0, out=None, accumulate=False):
    """``logoskg_embed_entities_backward``: the gradient [num_entities, dim] of ``embed_entities``'s table for ``dout``
    [*ids.shape, dim], that of its result; summed in 32 bits and rounded once; the same inputs give the same bits.

    ``out`` (of ``dout``'s type, or float32) takes it; with ``accumulate`` it is added to what stands there, and rows that no id
    names are not touched.  It shares no memory with ``dout``."""
    torch = _torch()
    device = _on_gpu(dout, "dout")
    if dout.dim() != ids.dim() + 1 or dout.shape[:-1] != ids.shape:
        raise ValueError(f"dout has the shape {tuple(dout.shape)}, and ids {tuple(ids.shape)}")
    dout_at, ids_at = _plain(dout, "dout", dout.dtype, device), _plain(ids, "ids", torch.int32, device)
    dim = dout.shape[-1]
    given = out is not None
    if not given:
        if accumulate:
            raise ValueError("accumulate needs out")
        out = dout.new_empty((num_entities, dim))
    if out.dtype is not dout.dtype and out.dtype is not torch.float32:
        raise ValueError("out must be of dout's type or float32")
    n, wide, row = _table(out, "out", out.dtype, device)
    if n != num_entities or wide != dim:
        raise ValueError(f"out has the shape {tuple(out.shape)}, not {(num_entities, dim)}")
    if given:
        _apart(out, "out", dout, ids)
    head = (104, device, _dtype(dout.dtype), _dtype(out.dtype), scale, 1 if accumulate else 0, ids.numel(), num_entities, dim, row,
            ids_at, dout_at, out.data_ptr())
    lib = _load()
    call = _embedding_grad_of(*head, 0, 0, 0)
    w = _workspace(lib.logoskg_embed_entities_backward_bytes(call), dout)
    _check(lib.logoskg_embed_entities_backward(call[:-24] + _last_of(*((0, 0) if w is None else (w.data_ptr(), w.numel())), _stream_handle(None, device))))
    return out


# ---------------------------------------------------------------- answers
def _answers(logits, target, mask, mask_row):
    """The first values of a _Policy (up to num_masks), its device, and the number of rows."""
    torch = _torch()
    if logits.dim() != 2:
        raise ValueError("logits must be [rows, vocab] with contiguous rows")
    (rows, vocab), (row, one) = logits.shape, logits.stride()
    if one != 1 and rows and vocab > 1:
        raise ValueError("logits must be [rows, vocab] with contiguous rows")
    device = _on_gpu(logits, "logits")
    words, masks = (vocab + 63) // 64, 0
    if mask is None:
        if mask_row is not None:
            raise ValueError("mask_row without a mask")
    else:
        masks = mask.shape[0] if mask.dim() == 2 else -1
        if masks == 0 and rows:
            raise ValueError("a mask without rows")
        _plain(mask, "mask", torch.int64, device, (masks if mask_row is not None else rows, words))
    head = (168, device, _dtype(logits.dtype), rows, vocab, row if rows > 1 else vocab, logits.data_ptr(),
            _plain(target, "target", torch.int32, device, (rows,)), 0 if mask is None else mask.data_ptr(),
            _plain(mask_row, "mask_row", torch.int32, device, (rows,)), masks)
    return head, device, rows


@_on_stream
def token_logp(logits, target, *, scale=1.0, mask=None, mask_row=None):
    """``logoskg_token_logp``: the log probabilities of the tokens ``target`` (int32 per row) under the softmax of
    ``scale`` x ``logits`` [rows, vocab] over the ids that a row's mask allows, as {"logp", "lse": float32 [rows]}.

    ``mask`` [masks, words] is ``entity_mask``'s, row i's is ``mask_row[i]`` (int32; None: mask i).  A target outside the
    vocabulary pads (logp 0); one that its mask hides has logp -inf.  A call without a gradient: what a policy has sampled by, or is
    kept near."""
    torch = _torch()
    head, device, rows = _answers(logits, target, mask, mask_row)
    logp, lse = (logits.new_empty((rows,), dtype=torch.float32) for _ in range(2))
    _check(_load().logoskg_token_logp(_policy_of(*head, scale, 0.0, 0.0, 0.0, 0, 0, 0, 0, logp.data_ptr(), lse.data_ptr(), 0, 0, 0,
                                                 _stream_handle(None, device))))
    return {"logp": logp, "lse": lse}


def _no_gradient(**tensors):
    """Refuses tensors whose gradient would be lost: what stands beside the rows is taken as it is."""
    for name, t in tensors.items():
        if t is not None and (t.requires_grad or _has_tangent(t)):
            raise ValueError(f"{name} requires a gradient, and policy_loss has none for it: detach it")


def _terms(advantage, old, ref, weight, clip, kl, scale, rows, device):
    """The values of a _Policy from scale to weight."""
    if kl and ref is None:
        raise ValueError("kl without ref")
    f = _torch().float32
    return (scale, kl, clip[0], clip[1], _plain(advantage, "advantage", f, device, (rows,)), _plain(old, "old", f, device, (rows,)),
            _plain(ref, "ref", f, device, (rows,)), _plain(weight, "weight", f, device, (rows,)))


@functools.lru_cache(None)
def _differentiable_policy():
    torch = _torch()

    class Policy(torch.autograd.Function):
        """``policy_loss`` of logits that require a gradient."""

        @staticmethod
        def forward(ctx, logits, target, advantage, tensors, kw):
            names = sorted(tensors)
            got = policy_loss(logits, target, advantage, **tensors, **kw)
            ctx.set_materialize_grads(False)
            ctx.save_for_backward(logits, target, advantage, got["lse"], *(tensors[n] for n in names))
            ctx.names, ctx.kw = names, kw
            ctx.mark_non_differentiable(got["logp"], got["lse"])
            return got["loss"], got["logp"], got["lse"]

        @staticmethod
        @torch.autograd.function.once_differentiable
        def backward(ctx, dloss, dlogp, dlse):
            if dloss is None:
                return (None,) * 5
            logits, target, advantage, lse, *rest = ctx.saved_tensors
            return (policy_loss_backward(dloss, logits, target, advantage, lse, **dict(zip(ctx.names, rest)), **ctx.kw),) + (None,) * 4

    return Policy


@_on_stream
def policy_loss(logits, target, advantage, *, old=None, ref=None, weight=None, clip=(0.2, 0.2), kl=0.0, scale=1.0, mask=None,
                mask_row=None, gradient=False):
    """``logoskg_policy_loss``: the clipped policy loss of sampled tokens with a KL term, as {"loss": float32 scalar, "logp",
    "lse": float32 [rows]}.

    Row by row, with ``token_logp``'s logp (which has the other arguments) and r = exp(logp - ``old``): the loss is ``weight`` times
    -min(r A, clamp(r, 1 - clip[0], 1 + clip[1]) A) + ``kl`` (exp(ref - logp) - (ref - logp) - 1), A = ``advantage``, summed over the rows.
    All of them are float32 per row; without ``old`` r is 1 (the samples are this policy's), without ``weight`` it is 1.  Rows whose target
    pads or is hidden, or whose weight is 0, do not count.  They are taken as they are: one that requires a gradient is refused (detach it).

    With ``gradient`` the same pass also returns "dlogits", the gradient of the loss with respect to ``logits`` in their type: for
    ``logits.backward(dlogits)``.  Without it, where ``logits`` requires a gradient, "loss" has one by ``policy_loss_backward``
    ("logp" and "lse" have none)."""
    torch = _torch()
    if torch.is_grad_enabled() and not gradient:
        _no_gradient(advantage=advantage, old=old, ref=ref, weight=weight)
    if not gradient and (logits.requires_grad and torch.is_grad_enabled() or _has_tangent(logits)):
        tensors = {n: t for n, t in dict(old=old, ref=ref, weight=weight, mask=mask, mask_row=mask_row).items() if t is not None}
        loss, logp, lse = _differentiable_policy().apply(logits, target, advantage, tensors, dict(clip=clip, kl=kl, scale=scale))
        return {"loss": loss, "logp": logp, "lse": lse}
    head, device, rows = _answers(logits, target, mask, mask_row)
    terms = _terms(advantage, old, ref, weight, clip, kl, scale, rows, device)
    loss, logp, lse = logits.new_empty((), dtype=torch.float32), logits.new_empty((rows,), dtype=torch.float32), logits.new_empty((rows,), dtype=torch.float32)
    dlogits = logits.new_empty(logits.shape) if gradient else None
    _check(_load().logoskg_policy_loss(_policy_of(*head, *terms, logp.data_ptr(), lse.data_ptr(), loss.data_ptr(),
                                                  0 if dlogits is None else dlogits.data_ptr(), 0, _stream_handle(None, device))))
    got = {"loss": loss, "logp": logp, "lse": lse}
    return got if dlogits is None else got | {"dlogits": dlogits}


@_on_stream
def policy_loss_backward(dloss, logits, target, advantage, lse, *, old=None, ref=None, weight=None, clip=(0.2, 0.2), kl=0.0, scale=1.0,
                         mask=None, mask_row=None):
    """``logoskg_policy_loss_backward``: the gradient of ``logits`` for ``dloss`` (float32 scalar on the device), that of
    ``policy_loss``'s "loss"; the other arguments are that call's, and its "lse".  Rows whose lse is 44 or more from 0 are read once more
    than others: what 32 bits of it do not hold is made again."""
    torch = _torch()
    head, device, rows = _answers(logits, target, mask, mask_row)
    terms = _terms(advantage, old, ref, weight, clip, kl, scale, rows, device)
    lse_at, dloss_at = _plain(lse, "lse", torch.float32, device, (rows,)), _plain(dloss, "dloss", torch.float32, device, ())
    dlogits = logits.new_empty(logits.shape)
    _check(_load().logoskg_policy_loss_backward(_policy_of(*head, *terms, 0, lse_at, 0, dlogits.data_ptr(), dloss_at,
                                                           _stream_handle(None, device))))
    return dlogits


# ---------------------------------------------------------------- the end of a step
_gradient_of = struct.Struct("=QQqii").pack


def _transposed(t) -> bool:
    return t.dim() == 2 and t.stride(0) == 1 and t.stride(1) == t.shape[0]


@_on_stream
def clip_gradients(grads, max_norm, *, scale=1.0, out=None):
    """``logoskg_clip_gradients``: multiplies ``grads`` (float32, bfloat16 and float16 tensors on one GPU, contiguous ones or transposes of
    such; None among them is left out) by ``scale``, and by ``max_norm`` / norm where the norm of all of them together, ``scale``
    included, is larger; returns that norm (float32 scalar on the device).

    In place, or into ``out``, one tensor per gradient in any of the three types (float32 for an optimizer that keeps 32 bits, say).  Sums are
    64-bit, and the same inputs give the same bits.  A norm that is not finite shows in the result: infinite, it makes zeros of the finite
    gradients (where all are finite and their norm is above float32's range, it shows as infinite, and they are scaled as others); NaN, NaN of all.  Tensors may not share memory."""
    torch = _torch()
    grads = list(grads)
    out = grads if out is None else list(out)
    if len(out) != len(grads):
        raise ValueError(f"{len(out)} outputs for {len(grads)} gradients")
    device, entries = -1, []
    for g, o in zip(grads, out):
        if g is None:
            continue
        if device < 0:
            device, like = _on_gpu(g, "a gradient"), g
        whole, dtype = g.is_contiguous(), g.dtype
        if g.get_device() != device or not (whole or _transposed(g)):
            raise ValueError(f"gradients must be contiguous tensors on cuda:{device}")
        kind = to = _dtype(dtype)
        if o is not g:
            if o is None or o.get_device() != device or o.shape != g.shape or not (o.is_contiguous() if whole else o.stride() == g.stride()):
                raise ValueError("an output must be laid out as its gradient")
            if o.dtype is not dtype:
                to = _dtype(o.dtype)
        entries.append(_gradient_of(g.data_ptr(), o.data_ptr(), g.numel(), kind, to))
    if device < 0:
        raise ValueError("no gradients")
    packed = b"".join(entries)
    norm = like.new_empty((), dtype=torch.float32)
    lib = _load()
    w = _workspace(lib.logoskg_clip_gradients_bytes(packed, len(entries)), like)
    _check(lib.logoskg_clip_gradients(device, packed, len(entries), max_norm, scale, norm.data_ptr(), w.data_ptr(), w.numel(),
                                      _stream_handle(None, device)))
    return norm
