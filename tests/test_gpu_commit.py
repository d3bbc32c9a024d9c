"""Commit of accepted rows, byte for byte (GPU): every cache kind, page sizes,
paths that overlap their own targets, entries and pages that fit nothing, caches
past 2^32 bytes, graphs; and a whole speculative step against a plain one."""
import numpy as np
import pytest
import torch

import speculate_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda"


def commit(kind, caches, page_size, table, num_pages, ctx, path, keep, new_lens=True):
    from paper_2609_36760_amd import _speculate as ms
    fn = ms.mla_bf16_commit if kind == "bf16" else ms.mla_lowbit_commit
    ctx = torch.tensor(ctx, dtype=torch.int32, device=DEV)
    lens = torch.full_like(ctx, -3) if new_lens else None
    fn(ref.library_format(kind, page_size), ms.layer_caches(caches), num_pages, torch.from_numpy(table).to(DEV), ctx,
       torch.tensor(path, dtype=torch.int32, device=DEV), torch.tensor(keep, dtype=torch.int32, device=DEV), lens)
    torch.cuda.synchronize()
    return None if lens is None else lens.cpu().numpy()


def random_caches(seed, layers, size):
    g = torch.Generator().manual_seed(seed)
    return [torch.randint(0, 256, (size,), generator=g, dtype=torch.uint8).to(DEV) for _ in range(layers)]


def padded(paths, most):
    return [p + [-1] * (most - len(p)) for p in paths]


@pytest.mark.parametrize("page_size", [32, 64, 96])
@pytest.mark.parametrize("kind", ref.KINDS)
def test_bytes(kind, page_size):
    rng = np.random.default_rng(page_size)
    most, layers = 64, 3
    ctx = [0, 1, 31, 62, 63, 100, 190, 200]
    paths = [[0], [0, 2, 5, 9], [0, 1, 2, 3], [5, 4, 3, 2, 1, 0], [], [0, 63], sorted(rng.choice(64, 40, replace=False).tolist()),
             rng.permutation(64).tolist()]
    table, num_pages = ref.block_table(rng, [c + 64 for c in ctx], page_size)
    caches = random_caches(7, layers, num_pages * ref.page_bytes(kind, page_size))
    before = np.stack([c.cpu().numpy() for c in caches])
    keep = [len(p) for p in paths]
    lens = commit(kind, caches, page_size, table, num_pages, ctx, padded(paths, most), keep)
    want, want_lens = ref.commit(before, kind, page_size, table, num_pages, ctx, padded(paths, most), keep, most)
    assert np.array_equal(np.stack([c.cpu().numpy() for c in caches]), want)
    assert lens.tolist() == want_lens.tolist()
    # twice the same input path on the moved rows, without the new lengths
    commit(kind, caches, page_size, table, num_pages, ctx, padded(paths, most), keep, new_lens=False)
    want, _ = ref.commit(want, kind, page_size, table, num_pages, ctx, padded(paths, most), keep, most)
    assert np.array_equal(np.stack([c.cpu().numpy() for c in caches]), want)


@pytest.mark.parametrize("kind", ["c4", "bf16"])
def test_entries_and_pages_that_fit_nothing(kind):
    rng = np.random.default_rng(2)
    most = 7
    ctx = [100, 60, 64 * 5 - 3, 20, 10]
    paths = [[0, -4, 2 ** 31 - 1, 6, 7, 3], [0, 2], [0, 4, 5], [0, 2, 3], [0, 3]]
    table, num_pages = ref.block_table(rng, [c + most for c in ctx], 64)
    table = np.ascontiguousarray(table[:, :5])          # positions past the page table
    table[3, 0] = num_pages
    table[4, 0] = -1
    caches = random_caches(3, 2, num_pages * ref.page_bytes(kind))
    before = np.stack([c.cpu().numpy() for c in caches])
    keep = [6, 2, 3, 3, 2]
    for k in (keep, [2 ** 31 - 1, -5, 0, 3, 99]):
        lens = commit(kind, caches, 64, table, num_pages, ctx, padded(paths, most), k)
        before, want = ref.commit(before, kind, 64, table, num_pages, ctx, padded(paths, most), k, most)
        assert np.array_equal(np.stack([c.cpu().numpy() for c in caches]), before)
        assert lens.tolist() == want.tolist()


def test_a_large_cache():
    """Rows past 2^32 bytes."""
    pages = (1 << 32) // 20736 + 50
    cache = torch.zeros(pages * 20736, dtype=torch.uint8, device=DEV)
    tail = cache[-20 * 20736:]
    tail.copy_(random_caches(4, 1, tail.numel())[0])
    before = tail.cpu().numpy()
    table = np.arange(20, dtype=np.int32).reshape(2, 10)
    ctx, paths = [60, 300], padded([[0, 3, 9], [0, 1, 7, 8, 60]], 64)
    commit("c4", [cache], 64, table + np.int32(pages - 20), pages, ctx, paths, [3, 5])
    want, _ = ref.commit(before[None], "c4", 64, table, 20, ctx, paths, [3, 5], 64)
    assert np.array_equal(tail.cpu().numpy(), want[0])


def test_a_graph():
    from paper_2609_36760_amd import _speculate as ms
    rng = np.random.default_rng(5)
    table, num_pages = ref.block_table(rng, [80, 120], 64)
    caches = random_caches(6, 2, num_pages * ref.page_bytes("c2p"))
    layers = ms.layer_caches(caches)
    host = np.stack([c.cpu().numpy() for c in caches])
    args = [torch.tensor(x, dtype=torch.int32, device=DEV) for x in ([60, 100], [[0, 2, 5], [0, 3, -1]], [3, 2], [0, 0])]
    block = torch.from_numpy(table).to(DEV)

    def call():
        ms.mla_lowbit_commit(ref.library_format("c2p"), layers, num_pages, block, *args)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for path, keep in (([[0, 2, 5], [0, 3, -1]], [3, 2]), ([[0, 1, 7], [0, 9, 12]], [3, 3]), ([[0, -1, -1], [1, -1, -1]], [1, 1])):
        args[1].copy_(torch.tensor(path, dtype=torch.int32))
        args[2].copy_(torch.tensor(keep, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        host, lens = ref.commit(host, "c2p", 64, table, num_pages, [60, 100], path, keep, 3)
        assert np.array_equal(np.stack([c.cpu().numpy() for c in caches]), host) and args[3].tolist() == lens.tolist()


@pytest.mark.parametrize("kind", ["c4", "c2p", "bf16"])
def test_whole_steps(kind):
    """Steps in a loop without the host: drafted rows appended, attended, verified, committed.  The cache then holds
    what a plain writer gives for the accepted tokens, and the attention of an accepted node equals, within both
    calls' bounds, the one of the same token in a cache that holds only its ancestors."""
    from paper_2609_36760_amd import _binding as mb
    from paper_2609_36760_amd import _speculate as ms
    rng = np.random.default_rng(8)
    g = torch.Generator().manual_seed(8)
    B, H, V, n, steps, first = 3, 16, 200, 7, 4, [40, 0, 61]
    most_len = max(first) + steps * n
    table, num_pages = ref.block_table(rng, [most_len] * B, 64)
    fmt, size = ref.library_format(kind), ref.page_bytes(kind)
    block = torch.from_numpy(table).to(DEV)
    append = mb.mla_bf16_append if kind == "bf16" else mb.mla_lowbit_quant_append
    attend = ms.mla_bf16_tree_attn if kind == "bf16" else ms.mla_lowbit_tree_attn
    move = ms.mla_bf16_commit if kind == "bf16" else ms.mla_lowbit_commit
    caches = [torch.zeros(num_pages * size, dtype=torch.uint8, device=DEV) for _ in range(2)]
    layers = ms.layer_caches(caches)
    truth = [[torch.randn((first[b], 576), generator=g).bfloat16() for b in range(B)] for _ in caches]

    def slots(b, positions):
        p = np.asarray(positions, np.int64)
        return table[b, p // 64].astype(np.int64) * 64 + p % 64

    for layer, cache in enumerate(caches):
        x = torch.cat(truth[layer]).to(DEV)
        s = np.concatenate([slots(b, np.arange(first[b])) for b in range(B)])
        append(fmt, x[:, :512].contiguous(), x[:, 512:].contiguous(), torch.from_numpy(s).to(DEV), cache, num_pages)
    ctx = torch.tensor(first, dtype=torch.int32, device=DEV)
    cu = torch.arange(B + 1, dtype=torch.int32, device=DEV) * n
    split = 64
    indptr, total = mb.mla_plan_splits(np.full(B, most_len, np.int32), split)       # one plan for every step
    plan = dict(split_tokens=split, split_indptr=torch.from_numpy(indptr).to(DEV), num_splits=total,
                workspace=torch.empty(ms.mla_tree_workspace_bytes(total, n, H), dtype=torch.uint8, device=DEV))
    path, out_tokens = (torch.zeros((B, n), dtype=torch.int32, device=DEV) for _ in range(2))
    keep, lens = torch.zeros(B, dtype=torch.int32, device=DEV), torch.zeros(B, dtype=torch.int32, device=DEV)
    space = torch.empty(ms.mla_verify_workspace_bytes(B * n, B, V), dtype=torch.uint8, device=DEV)
    kept_more = 0
    for step in range(steps):
        trees = [ref.random_tree(rng, n) for _ in range(B)]
        parents = torch.tensor(sum(trees, []), dtype=torch.int32, device=DEV)
        mask = ref.mask_tensor(sum((ref.lineage_masks(t) for t in trees), []), DEV)
        new = [torch.randn((B * n, 576), generator=g).bfloat16() for _ in caches]
        q = torch.randn((B * n, H, 576), generator=g).bfloat16().to(DEV)
        out = torch.zeros((B * n, H, 512), dtype=torch.bfloat16, device=DEV)
        pos = (ctx[:, None] + torch.arange(n, device=DEV, dtype=torch.int32)).long()
        slot = (block.long().gather(1, pos // 64) * 64 + pos % 64).reshape(-1)
        for layer, cache in enumerate(caches):
            x = new[layer].to(DEV)
            append(fmt, x[:, :512].contiguous(), x[:, 512:].contiguous(), slot, cache, num_pages)
            attend(fmt, q[..., :512].contiguous(), q[..., 512:].contiguous(), cache, num_pages, block, ctx, cu, mask, n, ref.TAU, out, **plan)
        logits = torch.randn((B * n, V), generator=g) * 0.5
        tokens = torch.randint(0, V, (B * n,), generator=g)
        for b in range(B):                              # drafts that are often taken
            for i in range(1, n):
                logits[b * n + trees[b][i], tokens[b * n + i]] += 5.0
        ms.mla_verify_tree(logits.to(DEV), tokens.to(torch.int32).to(DEV), parents, cu, n, torch.rand(B * n, generator=g).to(DEV),
                           torch.rand(B, generator=g).to(DEV), path, out_tokens, keep, space)
        move(fmt, layers, num_pages, block, ctx, path, keep, lens)
        old = ctx.cpu().numpy()
        ctx = lens.clone()
        # the accepted nodes' rows, and their attention over a cache of their own
        got = out.float().cpu().numpy()
        for b in range(B):
            nodes = path[b, :int(keep[b])].tolist()
            kept_more += len(nodes) - 1
            for layer in range(len(caches)):
                truth[layer][b] = torch.cat([truth[layer][b], new[layer][[b * n + i for i in nodes]]])
            if not nodes:
                continue
            own = torch.zeros(num_pages * size, dtype=torch.uint8, device=DEV)
            x = truth[-1][b].to(DEV)
            append(fmt, x[:, :512].contiguous(), x[:, 512:].contiguous(), torch.from_numpy(slots(b, np.arange(len(x)))).to(DEV), own, num_pages)
            values = ref.cached_values(own.cpu().numpy(), kind, table[b], len(x))
            rows = [b * n + i for i in nodes]
            want = ref.TreeRows(q[rows].double().cpu().numpy(), values, int(old[b]), ref.lineage_masks(ref.chain(len(nodes))), kind)
            want.check(got[rows], None, f"step {step}, sequence {b}")
            for layer, cache in enumerate(caches):
                x = truth[layer][b].to(DEV)
                fresh = torch.zeros(num_pages * size, dtype=torch.uint8, device=DEV)
                append(fmt, x[:, :512].contiguous(), x[:, 512:].contiguous(), torch.from_numpy(slots(b, np.arange(len(x)))).to(DEV), fresh, num_pages)
                a, c = (ref.cached_values(t.cpu().numpy(), kind, table[b], len(x)) for t in (fresh, cache))
                assert np.array_equal(a, c), f"step {step}, sequence {b}, layer {layer}"
    assert kept_more >= steps * B // 2
