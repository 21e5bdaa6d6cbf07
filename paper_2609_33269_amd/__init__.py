"""MI355X-native Action-Subspace-Protected (ASP) W4A4 linear layer of Q-WAM.

The compute lives in libqwam.so (hand-written HIP kernels for gfx950 behind a
C ABI, include/qwam.h).  `qwam` is its thin ctypes binding, `block` that of the
norms around a block and of the paged key-value cache, `calib` builds a
layer's factors offline, `inputs` draws the seeded synthetic workloads.
"""
from .block import (PagedCache, block_norm, block_norm_backward, kv_append, new_cache, paged_attention)  # noqa: F401
from .qwam import (PackedLayer, QwamError, aog_accumulate, aog_protected_basis,  # noqa: F401
                   aog_protected_basis_workspace, asp_layer, asp_linear, asp_matvec, debug_group_partials, forward, lib,
                   make_layer, make_plain_layer, pack_weights, quantize_act, quantize_act_deflated)

__all__ = ["PackedLayer", "PagedCache", "QwamError", "aog_accumulate", "aog_protected_basis", "aog_protected_basis_workspace",
           "asp_layer", "asp_linear", "asp_matvec", "block_norm", "block_norm_backward", "debug_group_partials", "forward",
           "kv_append", "lib", "make_layer", "make_plain_layer", "new_cache", "pack_weights", "paged_attention",
           "quantize_act", "quantize_act_deflated"]
