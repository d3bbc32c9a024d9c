"""ctypes binding of the speculative step's functions of ``libmla_lowbit.so``
(declared in include/mla_speculate.h).

As ``_prefill``: argument marshalling only, the names of the C entry points,
:class:`~._binding.MlaError` on a non-zero status, torch's current stream by
default; a call checks on the host that the tensors' sizes and types agree
(``ValueError``) and that they are on the current device.
"""
from __future__ import annotations

import ctypes

import torch

from . import _binding as mb
from ._prefill import BF16, D_C, D_R, F32, I32, I64, _cache, _int32s, _ints, _need, _on_device

SYMBOLS = (
    "mla_tree_split_tokens", "mla_tree_split_tokens_for", "mla_tree_workspace_bytes", "mla_lowbit_tree_attn", "mla_bf16_tree_attn",
    "mla_verify_workspace_bytes", "mla_verify_tree", "mla_lowbit_commit", "mla_bf16_commit",
)

MLA_LOGITS_BF16, MLA_LOGITS_FP32 = 0, 1
MAX_NODES = 64
MASKS = (torch.int64, torch.uint64)

_lib = None


def library() -> ctypes.CDLL:
    """The HIP library with the signatures of mla_speculate.h."""
    global _lib
    if _lib is not None:
        return _lib
    lib = mb.library()
    P, I, L, F, INT = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_int
    attn = [P, P, P, P, L, P, I, P, P, P, I, I, I, I, F, I, P, I, P, P, P, L, P]
    commit = [P, P, I, L, P, I, P, P, P, I, I, P, P]
    sig = {
        "mla_tree_split_tokens": (I, [P, I, I, I]),
        "mla_tree_split_tokens_for": (I, [P, P, I, I, I]),
        "mla_tree_workspace_bytes": (L, [I, I, I]),
        "mla_lowbit_tree_attn": (INT, attn),
        "mla_bf16_tree_attn": (INT, attn),
        "mla_verify_workspace_bytes": (L, [I, I, I]),
        "mla_verify_tree": (INT, [P, I, L, I, P, L, P, P, P, I, I, I, P, P, P, P, P, P, P, P, L, P]),
        "mla_lowbit_commit": (INT, commit),
        "mla_bf16_commit": (INT, commit),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _lib = lib
    return lib


def mla_tree_split_tokens(seq_lens, max_nodes: int, H: int) -> int:
    """Split size (0: unsplit) for sequences of ``seq_lens`` tokens, drafted
    ones included, whose node counts are not known; ``mla_plan_splits`` makes
    the plan."""
    lens = _int32s(seq_lens)
    _need(lens.ndim == 1, "seq_lens: one per sequence")
    n = library().mla_tree_split_tokens(lens.ctypes.data, lens.size, max_nodes, H)
    if n < 0:
        raise mb.MlaError("mla_tree_split_tokens", -n)
    return n


def mla_tree_split_tokens_for(seq_lens, nodes, max_nodes: int, H: int) -> int:
    """The same for sequences of ``nodes`` drafted tokens."""
    lens, counts = _int32s(seq_lens), _int32s(nodes)
    _need(lens.ndim == 1 and counts.shape == lens.shape, "seq_lens, nodes: one per sequence")
    n = library().mla_tree_split_tokens_for(lens.ctypes.data, counts.ctypes.data, lens.size, max_nodes, H)
    if n < 0:
        raise mb.MlaError("mla_tree_split_tokens_for", -n)
    return n


def _bytes(name: str, n: int) -> int:
    if n < 0:
        raise mb.MlaError(name, mb.MLA_EINVAL)
    return n


def mla_tree_workspace_bytes(num_splits: int, max_nodes: int, H: int) -> int:
    return _bytes("mla_tree_workspace_bytes", library().mla_tree_workspace_bytes(num_splits, max_nodes, H))


def mla_verify_workspace_bytes(num_nodes: int, B: int, vocab: int) -> int:
    return _bytes("mla_verify_workspace_bytes", library().mla_verify_workspace_bytes(num_nodes, B, vocab))


def _dense(t, shape, dtypes, what: str) -> None:
    if tuple(t.shape) != shape or t.dtype not in dtypes or not t.is_contiguous():
        raise ValueError(f"{what}: contiguous {list(shape)} of {dtypes}, got {tuple(t.shape)}, {t.dtype}")


def _table(block_table, B: int) -> None:
    if block_table.dim() != 2 or block_table.shape[0] != B or not block_table.is_contiguous() or block_table.dtype != I32:
        raise ValueError(f"block_table: contiguous int32 [{B}, max_pages]")


def _space(workspace) -> int:
    if workspace is None:
        return 0
    _need(workspace.is_contiguous(), "workspace: contiguous")
    return workspace.numel() * workspace.element_size()


def _tree_attn(name, page_bytes, fmt, q_lat, q_rope, cache, num_pages, block_table, ctx_lens, cu_nodes, tree_mask,
               max_nodes, softmax_scale, out, lse, split_tokens, split_indptr, num_splits, workspace, stream):
    _need(q_lat.dim() == 3, "q_lat: [nodes, H, 512]")
    T, H = q_lat.shape[0], q_lat.shape[1]
    B = ctx_lens.shape[0]
    _dense(q_lat, (T, H, D_C), BF16, "q_lat")
    _dense(q_rope, (T, H, D_R), BF16, "q_rope")
    _dense(out, (T, H, D_C), BF16, "out")
    if lse is not None:
        _dense(lse, (T, H), (F32,), "lse")
    _ints(ctx_lens, B, I32, "ctx_lens")
    _ints(cu_nodes, B + 1, I32, "cu_nodes")
    _dense(tree_mask, (T,), MASKS, "tree_mask")
    _cache(cache, page_bytes, num_pages)
    _table(block_table, B)
    if split_tokens:
        _need(split_indptr is not None, "split_indptr: needed with split_tokens")
        _ints(split_indptr, B + 1, I32, "split_indptr")
    size = _space(workspace)
    _on_device(q_lat, q_rope, cache, block_table, ctx_lens, cu_nodes, tree_mask, out, lse, split_indptr, workspace)
    mb._check(name, getattr(library(), name)(
        ctypes.byref(fmt), q_lat.data_ptr(), q_rope.data_ptr(), cache.data_ptr(), num_pages, block_table.data_ptr(),
        block_table.shape[1], ctx_lens.data_ptr(), cu_nodes.data_ptr(), tree_mask.data_ptr(), T, max_nodes, B, H,
        float(softmax_scale), split_tokens, mb._ptr(split_indptr), num_splits, out.data_ptr(), mb._ptr(lse),
        mb._ptr(workspace), size, mb._stream(stream)))


def mla_lowbit_tree_attn(fmt, q_lat, q_rope, cache, num_pages, block_table, ctx_lens, cu_nodes, tree_mask, max_nodes,
                         softmax_scale, out, lse=None, split_tokens=0, split_indptr=None, num_splits=0, workspace=None,
                         stream=None):
    """Attention of drafted tokens: queries ``q_lat`` [nodes, H, 512] and
    ``q_rope`` [nodes, H, 64] of all sequences' nodes, those of sequence b from
    ``cu_nodes[b]`` on and cached from position ``ctx_lens[b]`` on, into ``out``
    [nodes, H, 512] and ``lse`` fp32 [nodes, H].  ``tree_mask`` [nodes]: bit j,
    the node sees node j of its sequence."""
    _tree_attn("mla_lowbit_tree_attn", mb.mla_lowbit_page_bytes(fmt), fmt, q_lat, q_rope, cache, num_pages, block_table,
               ctx_lens, cu_nodes, tree_mask, max_nodes, softmax_scale, out, lse, split_tokens, split_indptr,
               num_splits, workspace, stream)


def mla_bf16_tree_attn(fmt, q_lat, q_rope, cache, num_pages, block_table, ctx_lens, cu_nodes, tree_mask, max_nodes,
                       softmax_scale, out, lse=None, split_tokens=0, split_indptr=None, num_splits=0, workspace=None,
                       stream=None):
    """The same over the BF16 cache."""
    _tree_attn("mla_bf16_tree_attn", mb.mla_bf16_page_bytes(fmt), fmt, q_lat, q_rope, cache, num_pages, block_table,
               ctx_lens, cu_nodes, tree_mask, max_nodes, softmax_scale, out, lse, split_tokens, split_indptr,
               num_splits, workspace, stream)


def _vocab_rows(t, T: int, V: int, what: str) -> int:
    """Stride of rows ``t`` [T, V] with unit stride in the last axis."""
    if tuple(t.shape) != (T, V) or (V > 1 and t.stride(1) != 1):
        raise ValueError(f"{what}: [{T}, {V}] rows with unit stride, got {tuple(t.shape)} strides {t.stride()}")
    return max(t.stride(0), V) if T < 2 else t.stride(0)


def mla_verify_tree(logits, tokens, parents, cu_nodes, max_nodes, u_accept, u_draw, path, out_tokens, keep, workspace,
                    temperature=None, draft_probs=None, logprobs=None, stream=None):
    """Verification of drafted ``tokens`` (trees by ``parents``) against
    ``logits`` (bf16 or fp32 [nodes, vocab]) with the random numbers ``u_accept``
    [nodes] and ``u_draw`` [B]: the nodes that stay into ``path`` [B, max_nodes],
    the emitted tokens into ``out_tokens``, their number into ``keep`` [B].
    ``draft_probs`` fp32 [nodes, vocab]: what every node's children were drawn
    from, independently of each other (None: fixed drafts, those drawn without
    replacement among them)."""
    _need(logits.dim() == 2, "logits: [nodes, vocab]")
    T, V = logits.shape
    B = u_draw.shape[0]
    _need(logits.dtype in (torch.bfloat16, F32), "logits: bf16 or fp32")
    stride = _vocab_rows(logits, T, V, "logits")
    q_stride = 0
    if draft_probs is not None:
        _need(draft_probs.dtype == F32, "draft_probs: fp32")
        q_stride = _vocab_rows(draft_probs, T, V, "draft_probs")
    _ints(tokens, T, I32, "tokens")
    _ints(parents, T, I32, "parents")
    _ints(cu_nodes, B + 1, I32, "cu_nodes")
    _ints(u_accept, T, F32, "u_accept")
    _ints(u_draw, B, F32, "u_draw")
    if temperature is not None:
        _ints(temperature, B, F32, "temperature")
    _dense(path, (B, max_nodes), (I32,), "path")
    _dense(out_tokens, (B, max_nodes), (I32,), "out_tokens")
    if logprobs is not None:
        _dense(logprobs, (B, max_nodes), (F32,), "logprobs")
    _ints(keep, B, I32, "keep")
    size = _space(workspace)
    _on_device(logits, tokens, parents, cu_nodes, u_accept, u_draw, path, out_tokens, keep, workspace, temperature,
               draft_probs, logprobs)
    mb._check("mla_verify_tree", library().mla_verify_tree(
        logits.data_ptr(), MLA_LOGITS_FP32 if logits.dtype == F32 else MLA_LOGITS_BF16, stride, V,
        mb._ptr(draft_probs), q_stride, tokens.data_ptr(), parents.data_ptr(), cu_nodes.data_ptr(), T, max_nodes, B,
        mb._ptr(temperature), u_accept.data_ptr(), u_draw.data_ptr(), path.data_ptr(), out_tokens.data_ptr(),
        mb._ptr(logprobs), keep.data_ptr(), mb._ptr(workspace), size, mb._stream(stream)))


class layer_caches:
    """The caches of a model's layers (tensors of one size on one device, each its
    own memory) as the table that the commit takes; keeps them alive."""

    def __init__(self, tensors):
        _need(len(tensors) > 0, "layer_caches: at least one")
        size = {t.numel() * t.element_size() for t in tensors}
        _need(len(size) == 1 and all(t.is_contiguous() for t in tensors), "layer_caches: contiguous, of one size")
        _need(len({t.device for t in tensors}) == 1, "layer_caches: on one device")
        _need(all(t.data_ptr() % 256 == 0 for t in tensors), "layer_caches: 256-byte aligned")
        self.tensors = list(tensors)
        self.bytes = size.pop()
        at = sorted(t.data_ptr() for t in tensors)
        _need(all(b - a >= max(self.bytes, 1) for a, b in zip(at, at[1:])), "layer_caches: each its own memory")
        self.table = torch.tensor([t.data_ptr() for t in tensors], dtype=I64, device=tensors[0].device)


def _commit(name, page_bytes, fmt, layers, num_pages, block_table, ctx_lens, path, keep, new_lens, stream):
    B = ctx_lens.shape[0]
    _need(path.dim() == 2, "path: [B, max_nodes]")
    _need(layers.bytes >= page_bytes * num_pages, "layers: smaller than num_pages pages")
    _ints(ctx_lens, B, I32, "ctx_lens")
    _dense(path, (B, path.shape[1]), (I32,), "path")
    _ints(keep, B, I32, "keep")
    _table(block_table, B)
    if new_lens is not None:
        _ints(new_lens, B, I32, "new_lens")
        at = new_lens.data_ptr() - path.data_ptr()
        _need(at <= -4 * B or at >= 4 * path.numel(), "new_lens: memory of its own")
    _on_device(layers.table, block_table, ctx_lens, path, keep, new_lens)
    mb._check(name, getattr(library(), name)(
        ctypes.byref(fmt), layers.table.data_ptr(), len(layers.tensors), num_pages, block_table.data_ptr(),
        block_table.shape[1], ctx_lens.data_ptr(), path.data_ptr(), keep.data_ptr(), path.shape[1], B,
        mb._ptr(new_lens), mb._stream(stream)))


def mla_lowbit_commit(fmt, layers, num_pages, block_table, ctx_lens, path, keep, new_lens=None, stream=None):
    """In every cache of ``layers`` (:class:`layer_caches`) the rows of the nodes
    that stay move up behind the context; ``new_lens`` = ``ctx_lens`` + ``keep``."""
    _commit("mla_lowbit_commit", mb.mla_lowbit_page_bytes(fmt), fmt, layers, num_pages, block_table, ctx_lens, path,
            keep, new_lens, stream)


def mla_bf16_commit(fmt, layers, num_pages, block_table, ctx_lens, path, keep, new_lens=None, stream=None):
    """The same in BF16 caches."""
    _commit("mla_bf16_commit", mb.mla_bf16_page_bytes(fmt), fmt, layers, num_pages, block_table, ctx_lens, path, keep,
            new_lens, stream)
