"""MI355X (gfx950) implementation of TransAct V2's lifelong-sequence serving
hot path: candidate-anchored NN select over the de-duplicated request-level
sequence, token gather and the fused-candidate causal encoder.

The compute lives in libtav2.so (HIP kernels behind the C ABI of
include/tav2.h); `paper_2506_02267_amd.tav2` is its thin Python binding.
"""
from . import tav2  # noqa: F401
from .tav2 import (DeviceCands, DeviceSeq, DeviceTokens, DeviceWeights, KvCache,  # noqa: F401
                   KvGroups, SelectEncode, Workspace, attend_window, beam_select, encode, gather,
                   kv_append, kv_attend, kv_attend_prefix, kv_compact, kv_extend, kv_fork, kv_free,
                   kv_reorder, kv_trim, load_library, nn_select, select_encode)
