"""The host side of mla_speculate.h: symbols, sizes, the split size, and refusals of
the C entry points and of the binding (CPU only; no GPU work is launched)."""
import ctypes
import math
import os
import re

import numpy as np
import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EINVAL, ENOTSUP = 1, 2


@pytest.fixture(scope="module")
def ms():
    from paper_2609_36760_amd import _binding, _speculate
    if not os.path.exists(_binding.LIB_PATH):
        pytest.skip("libmla_lowbit.so not built (run __graft_entry__.build())")
    _speculate.library()
    return _speculate


@pytest.fixture(scope="module")
def mb(ms):
    from paper_2609_36760_amd import _binding
    return _binding


def test_exports_every_declared_symbol(ms):
    text = open(os.path.join(ROOT, "include", "mla_speculate.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    assert sorted(set(re.findall(r"\b(mla_[a-z0-9_]+)\s*\(", text))) == sorted(ms.SYMBOLS)


def test_public_names(ms):
    import paper_2609_36760_amd as pkg
    for name in ms.SYMBOLS + ("layer_caches",):
        assert getattr(pkg, name) is getattr(ms, name)


def test_workspaces(ms, mb):
    assert ms.mla_tree_workspace_bytes(0, 1, 1) == 0
    assert ms.mla_tree_workspace_bytes(7, 8, 128) == 7 * 8 * 128 * (512 * 2 + 8)
    # 16 bytes for every chunk of 2 048 logits, 8 for every chunk and 4 for every sequence
    assert ms.mla_verify_workspace_bytes(5, 2, 2049) == 2 * (5 * 16 + 2 * 8) + 2 * 4
    assert ms.mla_verify_workspace_bytes(0, 0, 1) == 0
    for bad in ((-1, 1, 1), (1, 0, 1), (1, 65, 1), (1, 1, 0), (1, 64, (1 << 14) + 1)):
        with pytest.raises(mb.MlaError):
            ms.mla_tree_workspace_bytes(*bad)
    for bad in ((-1, 1, 1), (1, -1, 1), (1, 1, 0), (1, 1, (1 << 21) + 1)):
        with pytest.raises(mb.MlaError):
            ms.mla_verify_workspace_bytes(*bad)


def test_split_sizes(ms, mb):
    assert ms.mla_tree_split_tokens([74], 4, 16) == 0               # too short to share
    assert ms.mla_tree_split_tokens([], 4, 16) == 0
    assert ms.mla_tree_split_tokens([4000] * 64, 64, 128) == 0      # far more workgroups than compute units
    # even parts: 8 of 32 sequences of one row block, 4 of 8 sequences of 8 row blocks
    assert ms.mla_tree_split_tokens([4104] * 32, 8, 16) == 544
    assert ms.mla_tree_split_tokens([131136] * 8, 64, 16) == 32800
    for lens, n, H in (([1], 1, 1), ([2 ** 31 - 1], 64, 16), (list(range(1, 3000, 11)), 9, 128), ([5, 100000, 33], 3, 5)):
        s = ms.mla_tree_split_tokens(lens, n, H)
        assert s >= 0 and s % 32 == 0 and (s == 0 or s < max(lens) + 32)
    for bad in (([0], 1, 1), ([5, -1], 1, 1), ([5], 0, 1), ([5], 65, 1), ([5], 1, 0), ([5], 64, (1 << 14) + 1)):
        with pytest.raises(mb.MlaError):
            ms.mla_tree_split_tokens(*bad)
    assert ms.library().mla_tree_split_tokens(None, 1, 1, 1) == -EINVAL
    for bad in ([2 ** 31], [3.5], [-2 ** 32 + 5]):
        with pytest.raises((ValueError, OverflowError)):
            ms.mla_tree_split_tokens(bad, 1, 1)


def status(ms, name, base, over):
    args = dict(base)
    fmt = over.get("fmt", args.pop("fmt", None))
    args.pop("fmt", None)
    args.update({k: v for k, v in over.items() if k != "fmt"})
    head = [] if fmt is None else [ctypes.byref(fmt)] if fmt != "null" else [None]
    return getattr(ms.library(), name)(*head, *args.values(), None)


ATTN = dict(q_lat=256, q_rope=256, cache=256, num_pages=4, block_table=256, max_pages=2, ctx_lens=256, cu_nodes=256,
            mask=256, num_nodes=6, max_nodes=3, B=2, H=16, scale=0.07, split_tokens=64, split_indptr=256, num_splits=3,
            out=256, lse=None, workspace=256, workspace_bytes=3 * 3 * 16 * 1032)


@pytest.mark.parametrize("name", ["mla_lowbit_tree_attn", "mla_bf16_tree_attn"])
def test_attention_refusals(ms, mb, name):
    base = dict(ATTN, fmt=mb.cache_format())
    for key in ("q_lat", "q_rope", "cache", "block_table", "ctx_lens", "cu_nodes", "mask", "out", "split_indptr", "workspace"):
        assert status(ms, name, base, {key: None}) == EINVAL, key
    for over in (dict(B=-1), dict(num_nodes=-1), dict(num_pages=-1), dict(num_pages=0), dict(max_pages=0), dict(H=0), dict(max_nodes=0),
                 dict(scale=0.0), dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf), dict(split_tokens=-32),
                 dict(num_splits=-1), dict(cache=264), dict(workspace_bytes=3 * 3 * 16 * 1032 - 1), dict(fmt="null"),
                 dict(fmt=mb.cache_format(page_size=0))):
        assert status(ms, name, base, over) == EINVAL, over
    for over in (dict(max_nodes=65), dict(H=1 << 19), dict(split_tokens=48), dict(q_lat=264), dict(q_rope=264), dict(out=264),
                 dict(workspace=264), dict(max_pages=(1 << 24) + 1), dict(split_tokens=(1 << 30) + 32),
                 dict(num_splits=2 ** 31 - 1, max_nodes=64, H=1 << 14, workspace_bytes=2 ** 62),
                 dict(B=2 ** 31 - 1, max_nodes=64, H=128, split_tokens=0),
                 dict(fmt=mb.cache_format(d_c=256)), dict(fmt=mb.cache_format(page_size=48))):
        assert status(ms, name, base, over) == ENOTSUP, over
    # nothing to do: no pointer is looked at
    none = {k: None for k in ("q_lat", "q_rope", "cache", "block_table", "ctx_lens", "cu_nodes", "mask", "out", "split_indptr", "workspace")}
    assert status(ms, name, base, dict(none, B=0)) == 0
    assert status(ms, name, base, dict(none, num_nodes=0)) == 0
    if name == "mla_lowbit_tree_attn":
        assert status(ms, name, base, dict(fmt=mb.cache_format(c_bits=3))) == EINVAL


VERIFY = dict(logits=256, type=1, stride=100, vocab=100, probs=256, probs_stride=100, tokens=256, parents=256, cu_nodes=256,
              num_nodes=6, max_nodes=4, B=2, temperature=None, u_accept=256, u_draw=256, path=256, out_tokens=256,
              logprobs=None, keep=256, workspace=256, workspace_bytes=6 * 16 + 2 * 8 + 2 * 4)


def test_verification_refusals(ms):
    name = "mla_verify_tree"
    for key in ("logits", "tokens", "parents", "cu_nodes", "u_accept", "u_draw", "path", "out_tokens", "keep", "workspace"):
        assert status(ms, name, VERIFY, {key: None}) == EINVAL, key
    for over in (dict(type=2), dict(type=-1), dict(vocab=0), dict(stride=99), dict(probs_stride=99), dict(B=-1), dict(num_nodes=-1),
                 dict(max_nodes=0), dict(workspace_bytes=6 * 16 + 2 * 8 + 2 * 4 - 1)):
        assert status(ms, name, VERIFY, over) == EINVAL, over
    big = dict(stride=1 << 22, probs_stride=1 << 22, workspace_bytes=2 ** 62)
    for over in (dict(big, vocab=(1 << 21) + 1), dict(max_nodes=65), dict(B=65536, workspace_bytes=2 ** 62), dict(logits=258),
                 dict(type=0, logits=257), dict(probs=258), dict(workspace=264),
                 dict(big, vocab=1 << 21, B=65535, max_nodes=64)):
        assert status(ms, name, VERIFY, over) == ENOTSUP, over
    assert status(ms, name, VERIFY, dict(B=0, cu_nodes=None, path=None)) == 0


COMMIT = dict(caches=256, num_layers=3, num_pages=4, block_table=256, max_pages=2, ctx_lens=256, path=256, keep=256,
              max_nodes=4, B=2, new_lens=512)


@pytest.mark.parametrize("name", ["mla_lowbit_commit", "mla_bf16_commit"])
def test_commit_refusals(ms, mb, name):
    base = dict(COMMIT, fmt=mb.cache_format())
    for key in ("caches", "block_table", "ctx_lens", "path", "keep"):
        assert status(ms, name, base, {key: None}) == EINVAL, key
    for over in (dict(B=-1), dict(num_layers=-1), dict(num_pages=-1), dict(num_pages=0), dict(max_pages=0), dict(max_nodes=0),
                 dict(new_lens=256), dict(fmt="null"), dict(fmt=mb.cache_format(page_size=0))):
        assert status(ms, name, base, over) == EINVAL, over
    for over in (dict(max_nodes=65), dict(B=65536), dict(max_pages=(1 << 24) + 1), dict(num_layers=1 << 24, B=2048),
                 dict(fmt=mb.cache_format(d_r=32))):
        assert status(ms, name, base, over) == ENOTSUP, over
    assert status(ms, name, base, dict(B=0, ctx_lens=None, path=None, keep=None)) == 0
    assert status(ms, name, base, dict(num_layers=0, new_lens=None, ctx_lens=None)) == 0


def bf(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


def i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def test_binding_refuses_attention_tensors(ms, mb):
    fmt = mb.cache_format()
    good = dict(q_lat=bf(6, 4, 512), q_rope=bf(6, 4, 64), cache=torch.zeros(2 * 20736, dtype=torch.uint8), num_pages=2,
                block_table=i32(2, 3), ctx_lens=i32(2), cu_nodes=i32(3), tree_mask=torch.zeros(6, dtype=torch.int64), max_nodes=3,
                softmax_scale=0.07, out=bf(6, 4, 512))
    for over in (dict(q_lat=bf(6, 512)), dict(q_lat=bf(6, 4, 512).float()), dict(q_lat=bf(6, 4, 1024)[..., ::2]), dict(q_rope=bf(5, 4, 64)),
                 dict(q_rope=bf(6, 4, 64).half()), dict(out=bf(6, 4, 511)), dict(lse=torch.zeros(6, 5)), dict(ctx_lens=i32(2).long()),
                 dict(cu_nodes=i32(2)), dict(tree_mask=torch.zeros(7, dtype=torch.int64)), dict(tree_mask=i32(6)),
                 dict(cache=torch.zeros(2 * 20736 - 1, dtype=torch.uint8)), dict(block_table=i32(3, 3)), dict(block_table=i32(3, 2).T),
                 dict(split_tokens=64), dict(split_tokens=64, split_indptr=i32(2)),
                 dict(workspace=torch.zeros(8, dtype=torch.uint8)[::2])):
        with pytest.raises(ValueError):
            ms.mla_lowbit_tree_attn(fmt, **dict(good, **over))


def test_binding_refuses_verification_tensors(ms):
    f32 = torch.zeros
    good = dict(logits=f32(6, 50), tokens=i32(6), parents=i32(6), cu_nodes=i32(3), max_nodes=4, u_accept=f32(6), u_draw=f32(2),
                path=i32(2, 4), out_tokens=i32(2, 4), keep=i32(2), workspace=None)
    for over in (dict(logits=f32(6, 50).half()), dict(logits=f32(6)), dict(logits=f32(50, 6).T), dict(tokens=i32(5)), dict(parents=i32(6).long()),
                 dict(cu_nodes=i32(2)), dict(u_accept=f32(6).double()), dict(u_draw=f32(3)), dict(path=i32(2, 3)),
                 dict(out_tokens=i32(4, 2).T), dict(keep=i32(1)), dict(temperature=f32(3)), dict(logprobs=f32(2, 5)),
                 dict(draft_probs=f32(6, 49)), dict(draft_probs=bf(6, 50)), dict(workspace=torch.zeros(1).expand(4096))):
        with pytest.raises(ValueError):
            ms.mla_verify_tree(**dict(good, **over))


def test_binding_refuses_commit_tensors(ms, mb):
    with pytest.raises(ValueError):
        ms.layer_caches([])
    with pytest.raises(ValueError):
        ms.layer_caches([torch.zeros(256), torch.zeros(512)])
    with pytest.raises(ValueError):
        ms.layer_caches([torch.zeros(512)[::2]])
    whole = torch.zeros(1 << 16, dtype=torch.uint8)
    at = -whole.data_ptr() % 256
    with pytest.raises(ValueError):
        ms.layer_caches([whole[at + 16:at + 4112]])
    with pytest.raises(ValueError):         # a layer named twice would be moved twice, and layers may not overlap
        ms.layer_caches([whole[at:at + 20736]] * 2)
    with pytest.raises(ValueError):
        ms.layer_caches([whole[at:at + 20736], whole[at + 256:at + 20992]])
    layers = ms.layer_caches([whole[at:at + 20736], whole[at + 20992:at + 41728]])
    assert layers.table.tolist() == [whole.data_ptr() + at, whole.data_ptr() + at + 20992]
    good = dict(layers=layers, num_pages=1, block_table=i32(2, 3), ctx_lens=i32(2), path=i32(2, 4), keep=i32(2), new_lens=i32(2))
    for over in (dict(num_pages=2), dict(block_table=i32(1, 3)), dict(ctx_lens=i32(2).long()), dict(path=i32(8)), dict(path=i32(3, 4)),
                 dict(keep=i32(3)), dict(new_lens=i32(2, 1))):
        with pytest.raises(ValueError):
            ms.mla_lowbit_commit(mb.cache_format(), **dict(good, **over))
