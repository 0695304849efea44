"""MI355X-native batched k-hop knowledge-graph retrieval (LogosKG hot path).

The work is done by ``liblogoskg.so`` (hand-written HIP for gfx950, C ABI in
``include/logoskg.h``); this package is a thin ctypes binding with the same
names.  PyTorch is used only for device buffers and the stream handle.
"""
from .binding import (Graph, Result, LogosKGError, logoskg_build, logoskg_khop, logoskg_paths,
                      library_path, version)
from .reading import (attend, attend_backward, constrain_logits, distance_buckets, entity_mask, read_entities)
from .packed import pack_entities, packed_row_bytes, read_packed, unpack_entities
from .training import (clip_gradients, embed_entities, embed_entities_backward, policy_loss, policy_loss_backward, token_logp)

__all__ = ["Graph", "Result", "LogosKGError", "logoskg_build", "logoskg_khop", "logoskg_paths",
           "library_path", "version", "attend", "attend_backward", "constrain_logits", "distance_buckets",
           "entity_mask", "read_entities", "pack_entities", "packed_row_bytes", "read_packed", "unpack_entities", "clip_gradients",
           "embed_entities", "embed_entities_backward", "policy_loss", "policy_loss_backward", "token_logp"]
