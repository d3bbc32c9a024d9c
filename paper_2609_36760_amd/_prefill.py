"""ctypes binding of the prompt-side functions of ``libmla_lowbit.so``
(declared in include/mla_prefill.h).

As ``_binding``: argument marshalling only, the names of the C entry points,
:class:`~._binding.MlaError` on a non-zero status, torch's current stream by
default.  Sizes are taken from the tensors, so a call checks on the host that
they agree with each other (``ValueError``), and that the tensors are on the
current device.
"""
from __future__ import annotations

import ctypes

import numpy as np
import torch

from . import _binding as mb

SYMBOLS = (
    "mla_lowbit_norm_rope_append", "mla_bf16_norm_rope_append", "mla_lowbit_norm_rope_append_protected",
    "mla_rope_queries", "mla_lowbit_gather", "mla_bf16_gather", "mla_lowbit_gather_protected", "mla_plan_prefill",
    "mla_prefill_attn",
)

MLA_ROPE_PAIRS, MLA_ROPE_HALVES = 0, 1
D_C, D_R, D_NOPE, D_V = 512, 64, 128, 128
BF16 = (torch.bfloat16, torch.int16, torch.uint16)      # bf16 tensors, or their bit patterns
I32, I64, F32 = torch.int32, torch.int64, torch.float32


class mla_rotation(ctypes.Structure):
    _fields_ = [("table", ctypes.c_void_p), ("num_positions", ctypes.c_int64), ("layout", ctypes.c_int32)]


class mla_rms_norm(ctypes.Structure):
    _fields_ = [("weight", ctypes.c_void_p), ("eps", ctypes.c_float)]


class mla_prefill_plan(ctypes.Structure):
    _fields_ = [("plan_ints", ctypes.c_int64), ("workspace_bytes", ctypes.c_int64), ("total_q", ctypes.c_int64),
                ("total_kv", ctypes.c_int64), ("B", ctypes.c_int32), ("H", ctypes.c_int32),
                ("causal", ctypes.c_int32), ("rows", ctypes.c_int32), ("num_items", ctypes.c_int32),
                ("num_merges", ctypes.c_int32), ("num_parts", ctypes.c_int32), ("part_rows", ctypes.c_int32)]


class mla_head_rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("stride_t", ctypes.c_int64), ("stride_h", ctypes.c_int64)]


def rotation(table, layout: int = MLA_ROPE_PAIRS) -> mla_rotation:
    """``table``: fp32 [positions, 64], the cosines of the 32 pair angles, then
    their sines (kept alive by the result)."""
    _need(table.dim() == 2 and table.shape[1] == D_R and table.is_contiguous(), "table: [positions, 64], contiguous")
    _need(table.dtype == F32, "table: fp32")
    r = mla_rotation(table.data_ptr(), table.shape[0], layout)
    r.tensor = table
    return r


def rms_norm(eps: float = 1e-6, weight=None) -> mla_rms_norm:
    """``weight``: bf16 [512], or None (weightless)."""
    if weight is not None:
        _need(weight.dim() == 1 and weight.shape[0] == D_C and weight.is_contiguous() and weight.dtype in BF16,
              "weight: bf16 [512], contiguous")
    r = mla_rms_norm(None if weight is None else weight.data_ptr(), eps)
    r.tensor = weight
    return r


_lib = None


def library() -> ctypes.CDLL:
    """The HIP library with the signatures of mla_prefill.h."""
    global _lib
    if _lib is not None:
        return _lib
    lib = mb.library()
    P, I, L, F, INT = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_int
    append = [P, P, P, P, L, P, L, P, P, I, P, L]
    out = [P, L, P, L, P]
    read = [P, P, L, P, I, P, P, I, I]
    sig = {
        "mla_lowbit_norm_rope_append": append + out,
        "mla_bf16_norm_rope_append": append + out,
        "mla_lowbit_norm_rope_append_protected": [P] + append + [P, P, P, I, P, L] + out,
        "mla_rope_queries": [P, P, L, L, P, I, I, P, L, L, P],
        "mla_lowbit_gather": read + out,
        "mla_bf16_gather": read + out,
        "mla_lowbit_gather_protected": [P] + read + [P, P, L, P] + out,
        "mla_plan_prefill": [P, P, P, P, I, I, I, P, L, P],
        "mla_prefill_attn": [P, P, P, P, P, P, P, F, P, L, L, P, P, L, P],
    }
    for name, args in sig.items():
        fn = getattr(lib, name)
        fn.restype = INT
        fn.argtypes = args
    _lib = lib
    return lib


def _need(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


def _on_device(*tensors) -> None:
    """All tensors on the current device (whose current stream a call uses)."""
    here = torch.cuda.current_device()
    for t in tensors:
        if t is not None and t.get_device() != here:
            raise ValueError(f"a tensor is on {t.device}, the current device is cuda:{here}")


def _rows(t, n: int, width: int, what: str) -> None:
    """``t``: bf16 [n, width] with unit stride in the last axis."""
    if t.shape != (n, width) or t.stride(1) != 1 or t.dtype not in BF16:
        raise ValueError(f"{what}: bf16 [{n}, {width}] rows with unit stride, got {tuple(t.shape)} strides {t.stride()}")


def _ints(t, n: int, dtype, what: str) -> None:
    if t.shape != (n,) or t.dtype != dtype or not t.is_contiguous():
        raise ValueError(f"{what}: contiguous {dtype} [{n}], got {tuple(t.shape)}, {t.dtype}")


def _cache(cache, page_bytes: int, num_pages: int) -> None:
    if cache.numel() * cache.element_size() < page_bytes * num_pages or not cache.is_contiguous():
        raise ValueError("cache: smaller than num_pages pages")


def _dense(c_out, k_out, n):
    if c_out is not None:
        _rows(c_out, n, D_C, "c_out")
    if k_out is not None:
        _rows(k_out, n, D_R, "k_out")
    return (mb._ptr(c_out), D_C if c_out is None else c_out.stride(0),
            mb._ptr(k_out), D_R if k_out is None else k_out.stride(0))


def _append_args(page_bytes, norm, rot, c_kv, k_rope, positions, slot_mapping, cache, num_pages, c_out, k_out):
    n = c_kv.shape[0]
    _rows(c_kv, n, D_C, "c_kv")
    _rows(k_rope, n, D_R, "k_rope")
    _ints(positions, n, I32, "positions")
    _ints(slot_mapping, n, I64, "slot_mapping")
    _cache(cache, page_bytes, num_pages)
    _on_device(c_kv, k_rope, positions, slot_mapping, cache, rot.tensor, c_out, k_out,
               None if norm is None else norm.tensor)
    return (None if norm is None else ctypes.byref(norm), ctypes.byref(rot), c_kv.data_ptr(), c_kv.stride(0),
            k_rope.data_ptr(), k_rope.stride(0), positions.data_ptr(), slot_mapping.data_ptr(), n, cache.data_ptr(),
            num_pages), _dense(c_out, k_out, n)


def mla_lowbit_norm_rope_append(fmt, norm, rot, c_kv, k_rope, positions, slot_mapping, cache, num_pages, c_out=None,
                                k_out=None, stream=None):
    """Normalize (``norm`` None: not) and rotate the new tokens, quantize them
    into the cache, and store them as dense rows too (``c_out``, ``k_out``)."""
    a, o = _append_args(mb.mla_lowbit_page_bytes(fmt), norm, rot, c_kv, k_rope, positions, slot_mapping, cache,
                        num_pages, c_out, k_out)
    mb._check("mla_lowbit_norm_rope_append", library().mla_lowbit_norm_rope_append(
        ctypes.byref(fmt), *a, *o, mb._stream(stream)))


def mla_bf16_norm_rope_append(fmt, norm, rot, c_kv, k_rope, positions, slot_mapping, cache, num_pages, c_out=None,
                              k_out=None, stream=None):
    """The same into the BF16 cache."""
    a, o = _append_args(mb.mla_bf16_page_bytes(fmt), norm, rot, c_kv, k_rope, positions, slot_mapping, cache,
                        num_pages, c_out, k_out)
    mb._check("mla_bf16_norm_rope_append", library().mla_bf16_norm_rope_append(
        ctypes.byref(fmt), *a, *o, mb._stream(stream)))


def mla_lowbit_norm_rope_append_protected(fmt, policy, norm, rot, c_kv, k_rope, positions, slot_mapping, cache,
                                          num_pages, token_seq, seq_lens, prot_slot, prot, num_prot, c_out=None,
                                          k_out=None, stream=None):
    """The same under BF16 protection of sink and recent tokens."""
    a, o = _append_args(mb.mla_lowbit_page_bytes(fmt), norm, rot, c_kv, k_rope, positions, slot_mapping, cache,
                        num_pages, c_out, k_out)
    B = seq_lens.shape[0]
    _ints(token_seq, c_kv.shape[0], I32, "token_seq")
    _protection(fmt, policy, seq_lens, prot_slot, prot, num_prot, B)
    _on_device(token_seq, seq_lens, prot_slot, prot)
    mb._check("mla_lowbit_norm_rope_append_protected", library().mla_lowbit_norm_rope_append_protected(
        ctypes.byref(fmt), ctypes.byref(policy), *a, token_seq.data_ptr(), seq_lens.data_ptr(), prot_slot.data_ptr(),
        B, prot.data_ptr(), num_prot, *o, mb._stream(stream)))


def _protection(fmt, policy, seq_lens, prot_slot, prot, num_prot, B):
    _ints(seq_lens, B, I32, "seq_lens")
    _ints(prot_slot, B, I32, "prot_slot")
    if prot.numel() * prot.element_size() < num_prot * mb.mla_protect_buffer_bytes(fmt, policy) or not prot.is_contiguous():
        raise ValueError("prot: smaller than num_prot buffers")


def mla_rope_queries(rot, q, positions, out=None, stream=None):
    """Rotate the RoPE channels of queries ``q`` [n, H, 64] (a view with unit
    stride in the last axis) into ``out``, or in place."""
    out = q if out is None else out
    n, H = q.shape[0], q.shape[1]
    for t, what in ((q, "q"), (out, "out")):
        if t.dim() != 3 or t.shape[0] != n or t.shape[1] != H or t.shape[2] != D_R or t.stride(2) != 1 or t.dtype not in BF16:
            raise ValueError(f"{what}: bf16 [{n}, {H}, 64] rows with unit stride, got {tuple(t.shape)} strides {t.stride()}")
    _ints(positions, n, I32, "positions")
    _on_device(q, positions, out, rot.tensor)
    mb._check("mla_rope_queries", library().mla_rope_queries(
        ctypes.byref(rot), q.data_ptr(), q.stride(0), q.stride(1), positions.data_ptr(), n, H, out.data_ptr(),
        out.stride(0), out.stride(1), mb._stream(stream)))


def _read_args(page_bytes, cache, num_pages, block_table, cu_rows, first, c_out, k_out):
    B, n = block_table.shape[0], c_out.shape[0]
    _cache(cache, page_bytes, num_pages)
    if block_table.dim() != 2 or not block_table.is_contiguous() or block_table.dtype != I32:
        raise ValueError("block_table: contiguous int32 [B, max_pages]")
    _ints(cu_rows, B + 1, I32, "cu_rows")
    if first is not None:
        _ints(first, B, I32, "first")
    _on_device(cache, block_table, cu_rows, first, c_out, k_out)
    return (cache.data_ptr(), num_pages, block_table.data_ptr(), block_table.shape[1], mb._ptr(first),
            cu_rows.data_ptr(), B, n), _dense(c_out, k_out, n)


def mla_lowbit_gather(fmt, cache, num_pages, block_table, cu_rows, c_out, k_out, first=None, stream=None):
    """Tokens ``first[b] ..`` of every sequence as dense rows ``cu_rows[b] ..``
    of ``c_out`` [n, 512] and ``k_out`` [n, 64]."""
    a, o = _read_args(mb.mla_lowbit_page_bytes(fmt), cache, num_pages, block_table, cu_rows, first, c_out, k_out)
    mb._check("mla_lowbit_gather", library().mla_lowbit_gather(ctypes.byref(fmt), *a, *o, mb._stream(stream)))


def mla_bf16_gather(fmt, cache, num_pages, block_table, cu_rows, c_out, k_out, first=None, stream=None):
    a, o = _read_args(mb.mla_bf16_page_bytes(fmt), cache, num_pages, block_table, cu_rows, first, c_out, k_out)
    mb._check("mla_bf16_gather", library().mla_bf16_gather(ctypes.byref(fmt), *a, *o, mb._stream(stream)))


def mla_lowbit_gather_protected(fmt, policy, cache, num_pages, block_table, cu_rows, seq_lens, prot, num_prot,
                                prot_slot, c_out, k_out, first=None, stream=None):
    """The same, protected tokens from their bf16 rows."""
    a, o = _read_args(mb.mla_lowbit_page_bytes(fmt), cache, num_pages, block_table, cu_rows, first, c_out, k_out)
    _protection(fmt, policy, seq_lens, prot_slot, prot, num_prot, block_table.shape[0])
    _on_device(seq_lens, prot, prot_slot)
    mb._check("mla_lowbit_gather_protected", library().mla_lowbit_gather_protected(
        ctypes.byref(fmt), ctypes.byref(policy), *a, seq_lens.data_ptr(), prot.data_ptr(), num_prot,
        prot_slot.data_ptr(), *o, mb._stream(stream)))


def _int32s(x) -> np.ndarray:
    a = np.atleast_1d(np.asarray(x))
    with np.errstate(invalid="ignore"):
        b = np.ascontiguousarray(a, dtype=np.int32)
    _need(np.array_equal(a, b), "lengths and starts: whole numbers of 32 bits")
    return b


def mla_plan_prefill(q_lens, kv_lens, H: int, causal: bool = True, q_starts=None, kv_starts=None):
    """Host planner of the expanded attention: ``(plan int32, info)``.  The
    caller keeps a device copy of ``plan``; it serves every call with these
    lengths."""
    lens = [None if x is None else _int32s(x) for x in (q_lens, kv_lens, q_starts, kv_starts)]
    B = lens[0].size
    for x in lens:
        _need(x is None or (x.ndim == 1 and x.size == B), "lengths and starts: one per sequence")
    ptrs = [None if x is None else x.ctypes.data for x in lens]
    info = mla_prefill_plan()
    fn = library().mla_plan_prefill
    mb._check("mla_plan_prefill", fn(*ptrs, B, H, int(bool(causal)), None, 0, ctypes.byref(info)))
    plan = np.zeros(info.plan_ints, dtype=np.int32)
    mb._check("mla_plan_prefill", fn(*ptrs, B, H, int(bool(causal)), plan.ctypes.data, plan.size, ctypes.byref(info)))
    return plan, info


def _heads(t, rows: int, H: int, width: int, what: str) -> mla_head_rows:
    shape, strides = t.shape, t.stride()
    if len(shape) != 3 or shape[0] < rows or shape[1:] != (H, width) or strides[2] != 1 or t.dtype not in BF16:
        raise ValueError(f"{what}: bf16 [>= {rows}, {H}, {width}] rows with unit stride, got {tuple(shape)} strides {strides}")
    return mla_head_rows(t.data_ptr(), strides[0], strides[1])


def mla_prefill_attn(info, plan, q_nope, q_rope, k_nope, k_rope, v, softmax_scale, out, lse=None, workspace=None,
                     stream=None):
    """Expanded attention on a plan (``info`` from :func:`mla_plan_prefill`,
    ``plan`` its device copy): queries [rows, H, 128 | 64], keys [keys, H, 128]
    and [keys, 64], values [keys, H, 128] into ``out`` [rows, H, 128] and
    ``lse`` fp32 [rows, H].  ``workspace``: at least ``info.workspace_bytes``."""
    T, K, H = info.total_q, info.total_kv, info.H
    shape, strides = k_rope.shape, k_rope.stride()
    if len(shape) != 2 or shape[0] < K or shape[1] != D_R or strides[1] != 1 or k_rope.dtype not in BF16:
        raise ValueError(f"k_rope: bf16 [>= {K}, 64] rows with unit stride, got {tuple(shape)}")
    rows = (_heads(q_nope, T, H, D_NOPE, "q_nope"), _heads(q_rope, T, H, D_R, "q_rope"),
            _heads(k_nope, K, H, D_NOPE, "k_nope"), mla_head_rows(k_rope.data_ptr(), strides[0], 0),
            _heads(v, K, H, D_V, "v"))
    o = _heads(out, T, H, D_V, "out")
    _ints(plan, info.plan_ints, I32, "plan")
    if lse is not None and (lse.dim() != 2 or lse.shape[0] < T or lse.shape[1] != H or not lse.is_contiguous() or
                            lse.dtype != F32):
        raise ValueError(f"lse: contiguous fp32 [>= {T}, {H}], got {tuple(lse.shape)}")
    _need(workspace is None or workspace.is_contiguous(), "workspace: contiguous")
    _on_device(plan, q_nope, q_rope, k_nope, k_rope, v, out, lse, workspace)
    size = 0 if workspace is None else workspace.numel() * workspace.element_size()
    mb._check("mla_prefill_attn", library().mla_prefill_attn(
        ctypes.byref(info), plan.data_ptr(), *map(ctypes.byref, rows), float(softmax_scale), o.data,
        o.stride_t, o.stride_h, mb._ptr(lse), mb._ptr(workspace), size, mb._stream(stream)))
