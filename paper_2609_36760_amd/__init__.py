"""Low-bit MLA decode for AMD MI355X (gfx950).

The compute lives in ``libmla_lowbit.so`` (HIP kernels behind the C ABI of
include/mla_lowbit.h, include/mla_prefill.h and include/mla_speculate.h);
``_binding``, ``_prefill`` and ``_speculate`` forward to it with the same names.
``synthetic`` draws seeded inputs; ``runner`` sets up device buffers and
runs whole decode steps through the binding.  Importing this package does not
load the library; the first binding call does, and fails loudly if it is not
built.
"""
from __future__ import annotations

_BINDING_NAMES = (
    "MlaError", "cache_format", "library", "mla_lowbit_page_bytes", "mla_bf16_page_bytes",
    "mla_lowbit_quant_append", "mla_bf16_append", "mla_plan_splits", "mla_lowbit_decode_attn",
    "mla_bf16_decode_attn", "mla_splitkv_combine", "mla_status_str", "mla_last_hip_error", "SYMBOLS",
)
_PREFILL_NAMES = (
    "mla_lowbit_norm_rope_append", "mla_bf16_norm_rope_append", "mla_lowbit_norm_rope_append_protected",
    "mla_rope_queries", "mla_lowbit_gather", "mla_bf16_gather", "mla_lowbit_gather_protected", "mla_plan_prefill",
    "mla_prefill_attn", "rotation", "rms_norm", "MLA_ROPE_PAIRS", "MLA_ROPE_HALVES",
)
_SPECULATE_NAMES = (
    "mla_tree_split_tokens", "mla_tree_split_tokens_for", "mla_tree_workspace_bytes", "mla_lowbit_tree_attn",
    "mla_bf16_tree_attn", "mla_verify_workspace_bytes", "mla_verify_tree", "layer_caches", "mla_lowbit_commit", "mla_bf16_commit",
)


def __getattr__(name):
    if name in _BINDING_NAMES:
        from . import _binding
        return getattr(_binding, name)
    if name in _PREFILL_NAMES:
        from . import _prefill
        return getattr(_prefill, name)
    if name in _SPECULATE_NAMES:
        from . import _speculate
        return getattr(_speculate, name)
    raise AttributeError(name)
