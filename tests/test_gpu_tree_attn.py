"""Attention of drafted tokens against 64 bits (GPU): every cache kind, heads from
1 to 128, contexts from none to several splits, trees of 1 to 64 nodes, masks of
any kind, ragged batches, and what must not be touched."""
import math

import numpy as np
import pytest
import torch

import speculate_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda"


class Batch:
    """Sequences with contexts ``ctx`` and trees ``masks`` (one list per sequence), cached by the library's writer."""

    def __init__(self, seed, kind, H, ctx, masks, page_size=64, behind=0, strange=None, gain=1.0):
        from paper_2609_36760_amd import _binding as mb
        from paper_2609_36760_amd import _speculate as ms
        self.mb, self.ms = mb, ms
        rng = np.random.default_rng(seed)
        self.kind, self.H, self.ctx, self.masks, self.P = kind, H, ctx, masks, page_size
        self.nodes = [len(m) for m in masks]
        self.lens = [c + n for c, n in zip(ctx, self.nodes)]
        self.most = max(self.nodes + [1])
        self.table, self.num_pages = ref.block_table(rng, self.lens, page_size)
        self.fmt = ref.library_format(kind, page_size)
        self.cu = np.concatenate([[0], np.cumsum(self.nodes)]).astype(np.int32)
        self.T = int(self.cu[-1]) + behind
        g = torch.Generator().manual_seed(seed)
        total = sum(self.lens)
        x = torch.randn((total, 576), generator=g)
        x[:, torch.randperm(512, generator=g)[:5]] *= 6.0
        if strange is not None:             # (sequence, position) -> values of that row
            starts = np.concatenate([[0], np.cumsum(self.lens)])
            for (b, t), put in strange.items():
                put(x[int(starts[b]) + t])
        x = x.bfloat16()
        slots = np.concatenate([self.table[b, np.arange(n) // page_size].astype(np.int64) * page_size + np.arange(n) % page_size
                                for b, n in enumerate(self.lens)]) if total else np.zeros(0, np.int64)
        self.cache = torch.full((self.num_pages * ref.page_bytes(kind, page_size),), 0xA5, dtype=torch.uint8, device=DEV)
        if kind == "bf16":                  # unused rows hold NaN
            self.cache.view(torch.int16).fill_(0x7FC0)
        append = mb.mla_bf16_append if kind == "bf16" else mb.mla_lowbit_quant_append
        xd = x.to(DEV)
        if total:
            append(self.fmt, xd[:, :512].contiguous(), xd[:, 512:].contiguous(), torch.from_numpy(slots).to(DEV), self.cache, self.num_pages)
        self.q = (torch.randn((self.T, H, 576), generator=g) * gain).bfloat16()
        self.q_lat, self.q_rope = (t.contiguous().to(DEV) for t in (self.q[..., :512], self.q[..., 512:]))
        self.block_table = torch.from_numpy(self.table).to(DEV)
        self.ctx_d = torch.tensor(ctx, dtype=torch.int32, device=DEV)
        self.cu_d = torch.from_numpy(self.cu).to(DEV)
        self.mask = ref.mask_tensor([m for ms_ in masks for m in ms_] + [0] * behind, DEV)
        self.out = torch.full((self.T, H, 512), -77.0, dtype=torch.bfloat16, device=DEV)
        self.lse = torch.full((self.T, H), -77.0, device=DEV)

    def plan(self, split, lens=None):
        """Arguments of a split call (the plan for ``lens``: lengths that may be reached)."""
        if not split:
            return {}
        indptr, total = self.mb.mla_plan_splits(np.maximum(np.asarray(lens or self.lens, np.int32), 1), split)
        size = self.ms.mla_tree_workspace_bytes(total, self.most, self.H)
        return dict(split_tokens=split, split_indptr=torch.from_numpy(indptr).to(DEV), num_splits=total,
                    workspace=torch.full((size,), 0xFF, dtype=torch.uint8, device=DEV))

    def call(self, out=None, lse=None, stream=None, **plan):
        fn = self.ms.mla_bf16_tree_attn if self.kind == "bf16" else self.ms.mla_lowbit_tree_attn
        fn(self.fmt, self.q_lat, self.q_rope, self.cache, self.num_pages, self.block_table, self.ctx_d, self.cu_d, self.mask,
           self.most, ref.TAU, self.out if out is None else out, lse=self.lse if lse is None else lse, stream=stream, **plan)

    def check(self, split, bad=()):
        """``bad``: (sequence, position) of keys that are not finite."""
        torch.cuda.synchronize()
        cache = self.cache.cpu().numpy()
        out, lse = self.out.float().cpu().numpy(), self.lse.cpu().numpy()
        worst = 0.0
        for b, n in enumerate(self.nodes):
            a = int(self.cu[b])
            if n == 0:
                continue
            x = ref.cached_values(cache, self.kind, self.table[b], self.lens[b], self.P)
            want = ref.TreeRows(self.q[a:a + n].double().numpy(), x, self.ctx[b], self.masks[b], self.kind, split=bool(split),
                                bad=[t for s, t in bad if s == b])
            worst = max(worst, want.check(out[a:a + n], lse[a:a + n], f"sequence {b}"))
        end = int(self.cu[-1])
        assert (out[end:] == -77.0).all() and (lse[end:] == -77.0).all(), "rows behind the last node were written"
        return worst


def trees(seed, counts, how="tree"):
    rng = np.random.default_rng(seed)
    got = []
    for n in counts:
        if how == "any":                # any set of nodes, also none, also bits past the tree
            got.append([int(rng.integers(0, 1 << 62)) * int(rng.integers(0, 2)) for _ in range(n)])
        else:
            got.append(ref.lineage_masks(ref.chain(n) if how == "chain" else ref.random_tree(rng, n)) if n else [])
    return got


CASES = [
    # (heads, contexts, nodes, masks, split, page size)
    (16, [0], [1], "tree", 0, 64),
    (1, [5], [3], "tree", 0, 64),
    (16, [31, 32, 33], [4, 4, 4], "chain", 0, 64),
    (16, [100, 0, 257], [4, 2, 3], "tree", 64, 64),
    (5, [63, 1, 190], [13, 7, 1], "any", 32, 32),
    (20, [64, 65, 7], [9, 33, 64], "tree", 0, 96),
    (16, [200, 0, 31], [64, 40, 32], "any", 96, 64),
    (64, [300, 17], [13, 5], "tree", 128, 64),
    (128, [70, 0, 129, 500], [8, 0, 3, 1], "tree", 0, 64),
    (128, [1000, 3], [6, 2], "any", 256, 128),
    (48, [90, 40, 0, 0, 222], [0, 5, 0, 1, 21], "tree", 64, 64),
]


@pytest.mark.parametrize("kind", ref.KINDS)
@pytest.mark.parametrize("case", range(len(CASES)))
def test_against_64_bits(case, kind):
    H, ctx, nodes, how, split, P = CASES[case]
    b = Batch(100 + case, kind, H, ctx, trees(case, nodes, how), page_size=P, behind=3)
    b.call(**b.plan(split))
    print("of the bound:", b.check(split))


@pytest.mark.parametrize("kind", ["c4", "bf16"])
def test_a_plan_for_longer_sequences_and_a_repeated_call(kind):
    b = Batch(7, kind, 16, [40, 130, 0], trees(3, [5, 9, 2]), behind=2)
    plan = b.plan(64, lens=[600, 140, 333])
    b.call(**plan)
    b.check(64)
    out, lse = b.out.clone(), b.lse.clone()
    b.call(**plan)
    assert torch.equal(out.view(torch.int16), b.out.view(torch.int16)) and torch.equal(lse, b.lse)


@pytest.mark.parametrize("split", [0, 32])
@pytest.mark.parametrize("kind,H", [("bf16", 16), ("bf16", 64), ("c4", 16), ("c2p", 64)])
def test_hidden_keys_that_are_not_finite(kind, H, split):
    """Nodes 1 and 3 are not finite in some channel: those that see them are NaN, no other row is."""
    n, ctx = 6, 50
    strange = {}
    for t, value in ((ctx + 1, math.inf), (ctx + 3, math.nan)):
        def put(row, value=value, t=t):
            row[t % 512] = value
        strange[(0, t)] = put
    b = Batch(11, kind, H, [ctx, 20], [ref.lineage_masks([-1, 0, 0, 0, 1, 2]), ref.lineage_masks(ref.chain(3))], strange=strange)
    b.call(**b.plan(split))
    torch.cuda.synchronize()
    cache = b.cache.cpu().numpy()
    x = ref.cached_values(cache, kind, b.table[0], b.lens[0])
    bad = [(0, int(t)) for t in np.nonzero(~np.isfinite(x).all(1))[0]]
    assert {t for _, t in bad} <= {ctx + 1, ctx + 3} and (kind != "bf16" or len(bad) == 2)
    b.check(split, bad)


@pytest.mark.parametrize("kind,split,longer", [("c4", 0, 0), ("c4", 64, 0), ("bf16", 32, 40), ("c2p", 96, 500)])
def test_more_sequences_than_lanes(kind, split, longer):
    """70 sequences (the launch finds its work another way up to 64), a plan for longer ones too."""
    rng = np.random.default_rng(split)
    ctx = rng.integers(0, 200, 70).tolist()
    b = Batch(71, kind, 16, ctx, trees(6, rng.integers(0, 7, 70).tolist()), behind=2)
    b.call(**b.plan(split, lens=[n + longer for n in b.lens] if longer else None))
    b.check(split)


@pytest.mark.parametrize("n", [3, 70])
def test_more_splits_named_than_the_plan_has(n):
    """A call captured for the most splits serves a plan of fewer: the last sequence has one split here."""
    b = Batch(74, "c4", 16, [150] * (n - 1) + [20], trees(9, [4] * n), behind=1)
    plan = b.plan(64)
    plan["num_splits"] += 9
    plan["workspace"] = torch.full((b.ms.mla_tree_workspace_bytes(plan["num_splits"], b.most, b.H),), 255, dtype=torch.uint8, device=DEV)
    for _ in range(3):
        b.out.fill_(-77.0)
        b.call(**plan)
        b.check(64)


def test_as_many_sequences_as_lanes():
    rng = np.random.default_rng(1)
    b = Batch(72, "c4", 20, rng.integers(0, 300, 64).tolist(), trees(7, rng.integers(0, 9, 64).tolist()))
    for split in (0, 32, 128):
        b.out.fill_(-77.0)
        b.call(**b.plan(split, lens=[n + 50 for n in b.lens]))
        b.check(split)


def test_many_splits_of_few_sequences():
    """16 splits and more per sequence: the merge shares a row's splits between waves."""
    b = Batch(73, "c4", 16, [900, 40, 1500], trees(8, [9, 3, 30]), behind=1)
    b.call(**b.plan(32))
    b.check(32)


def test_large_scores_and_spread_weights():
    """Scores far from one another, in both directions along the keys: the reference has to move."""
    for gain in (8.0, 0.02):
        b = Batch(21, "c4", 16, [900, 64], trees(5, [8, 30]), gain=gain)
        b.call(**b.plan(256))
        b.check(256)


def test_another_stream_and_a_graph():
    from paper_2609_36760_amd import _speculate  # noqa: F401
    b = Batch(31, "c4", 16, [150, 77], trees(9, [8, 12]))
    plan = b.plan(64)
    b.call(**plan)
    b.check(64)
    want, want_lse = b.out.clone(), b.lse.clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b.out.fill_(0.0)
        b.call(**plan)
    s.synchronize()
    assert torch.equal(want, b.out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.call(**plan)
    for _ in range(3):
        b.out.fill_(1.0)
        b.lse.fill_(1.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(want, b.out) and torch.equal(want_lse, b.lse)
    # lengths are read on the device: a shorter context in the same graph
    b.ctx_d[0] = 100
    b.ctx[0], b.lens[0] = 100, 108
    graph.replay()
    torch.cuda.synchronize()
    b.check(64)


def test_a_chain_equals_causal_decode():
    """Two nodes in a chain are the two query tokens of a causal decode, bit for bit in workgroups of one shape."""
    b = Batch(41, "c4", 128, [333, 64, 40], [ref.lineage_masks(ref.chain(2))] * 3)
    b.call()
    b.check(0)
    out = torch.zeros((3, 2, 128, 512), dtype=torch.bfloat16, device=DEV)
    lse = torch.zeros((3, 2, 128), device=DEV)
    lens = torch.tensor(b.lens, dtype=torch.int32, device=DEV)
    b.mb.library().mla_internal_shape_next_decode(128, 4)
    b.mb.mla_lowbit_decode_attn(b.fmt, b.q_lat.view(3, 2, 128, 512), b.q_rope.view(3, 2, 128, 64), b.cache, b.num_pages,
                                b.block_table, lens, 2, 128, ref.TAU, out=out, lse=lse)
    assert torch.equal(out.view(6, 128, 512), b.out) and torch.equal(lse.view(6, 128), b.lse)


def test_a_long_cache():
    """Pages past 2^32 bytes of the cache, and a context of many tiles."""
    b = Batch(51, "c4", 16, [5000], trees(2, [7]))
    big = torch.empty((1 << 32) // 20736 + 200, 20736, dtype=torch.uint8, device=DEV)
    far = big.shape[0] - b.num_pages
    big[far:] = b.cache.view(-1, 20736)
    plan = b.plan(512)
    b.call(**plan)
    want = b.out.clone()
    b.out.fill_(0.0)
    small, pages, table = b.cache, b.num_pages, b.block_table
    b.cache, b.num_pages, b.block_table = big, big.shape[0], table + far
    b.call(**plan)
    assert torch.equal(want, b.out)
    b.cache, b.num_pages, b.block_table = small, pages, table
    b.check(512)


def test_device_values_out_of_range_stay_inside():
    """Page ids, lengths, node ranges and plans that fit nothing: every index is clamped, whatever comes out."""
    b = Batch(61, "c4", 16, [100, 40], trees(4, [6, 5]), behind=4)
    plan = b.plan(64)
    for change in (lambda: b.block_table.fill_(1 << 30), lambda: b.block_table.fill_(-5),
                   lambda: b.ctx_d.copy_(torch.tensor([1 << 30, -7], dtype=torch.int32)),
                   lambda: b.cu_d.copy_(torch.tensor([-3, 70, 9000], dtype=torch.int32)),
                   lambda: b.cu_d.copy_(torch.tensor([9, 2, 1], dtype=torch.int32)),
                   lambda: plan["split_indptr"].copy_(torch.tensor([2, 1 << 30, -1], dtype=torch.int32)),
                   lambda: b.mask.fill_(-1)):
        change()
        b.call(**plan)
        torch.cuda.synchronize()
