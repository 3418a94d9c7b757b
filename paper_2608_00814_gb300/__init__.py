"""GB300 (sm_103a) tree-verification step of OoO-Spec (arXiv 2608.00814).

The verify step -- one forward pass of the target over a packed candidate
tree with an ancestor mask, greedy longest-prefix acceptance, and KV
compaction -- runs entirely in the CUDA library built from csrc/ (C ABI in
include/oos.h).  `binding` marshals PyTorch tensors into that ABI.

For batches of requests behind one shared prompt the library also offers the
operators of a layer's step: oos_qk_norm_rope, oos_paged_append and
oos_shared_prefix_attention.
"""

from . import binding  # noqa: F401
from .binding import (Batch, KVCache, OosError, OosModel, OosRopeConfig, PagedCache, VerifyOutputs,  # noqa: F401
                      oos_accept_walk, oos_kv_compact, oos_last_status, oos_paged_append, oos_qk_norm_rope,
                      oos_shared_prefix_attention, oos_shared_prefix_attention_workspace_bytes, oos_status_string,
                      oos_tree_verify, oos_tree_verify_debug, oos_workspace_bytes, tree_verify)
