"""The operators of a speculative decode step, in their plain form and as the library's calls.

A drafting model proposes a tree of tokens behind every sequence; the target
model looks at all of them in one step:

* ``attn``: the absorbed attention of the drafted tokens' queries over the
  paged cache, which holds the context and, behind it, the drafted tokens
  themselves; a drafted token sees the context and its own ancestors;
* ``verify``: the drafted tokens are accepted or not by the target's logits and
  given random numbers, and the next token is drawn;
* ``commit``: the cached rows of the accepted tokens move up behind the context,
  in all layers' caches.

Heads per GPU 16, 64 and 128 (a 128-head layer under tensor parallelism),
64-token pages in random order, INT4 and INT2 content, both metadata formats and
the BF16 cache; vocabularies of 32K and 128K tokens and an odd one.

Sizes, lengths and the trees' shapes are part of a case and do not depend on the
seed.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda"
PAGE = 64
TAU = 1.0 / math.sqrt(192.0)
MOST_NODES = 64
MOST_PAIRS = 1 << 30            # (row, key) scores of an attention case
MOST_TOKENS = 1 << 20           # cached tokens of an attention case
MOST_LOGITS = 1 << 25
MOST_MOVES = 1 << 14            # (accepted token, layer) pairs of a commit case


def _attn(name, B, ctx, nodes, H, cache="c4", meta="fp16", lo=0, few=0, chain=False, shape=0):
    """``ctx``: context tokens (with ``lo`` the upper end of log-uniform lengths); ``nodes``: drafted tokens of every
    sequence, the root among them (with ``few`` the upper end)."""
    c = dict(op="attn", B=B, ctx=ctx, lo=lo, nodes=nodes, few=few, H=H, cache=cache, meta=meta, chain=chain, shape=shape)
    return dict(c, name=name) if name else c


def _verify(name, B, nodes, vocab, kind="bf16", sampled=False, few=0, chain=False, greedy="none", shape=0):
    """``sampled``: drafts drawn from given probabilities, else fixed ones; ``greedy``: none, some or all sequences."""
    c = dict(op="verify", B=B, nodes=nodes, few=few, vocab=vocab, kind=kind, sampled=sampled, chain=chain, greedy=greedy, shape=shape)
    return dict(c, name=name) if name else c


def _commit(name, B, nodes, layers, cache="c4", meta="fp16", few=0, shape=0):
    c = dict(op="commit", B=B, nodes=nodes, few=few, layers=layers, cache=cache, meta=meta, shape=shape)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the smallest call: a chat's first step with four drafted tokens, on one GPU of eight
        _attn("attn_h16_1x4_on_70", 1, 70, 4, 16, chain=True),
        # ordinary traffic on one GPU of eight
        _attn("attn_h16_32x8_on_4k", 32, 4096, 8, 16, shape=1),
        # all heads, contexts and trees of unequal, odd sizes
        _attn("attn_h128_24_ragged", 24, 16384, 32, 128, lo=1000, few=5, shape=2),
        # a large tree over long documents, in 2 bits and the paper's storage
        _attn("attn_h16_8x64_on_128k_int2", 8, 131072, 64, 16, cache="c2", meta="paper", shape=3),
        # the unquantized cache, an odd tree behind odd contexts
        _attn("attn_h64_24x13_on_3001_bf16", 24, 3001, 13, 64, cache="bf16", shape=4),
        # the smallest call: one greedy sequence, a chain of four behind the root
        _verify("verify_1x5_32k_greedy", 1, 5, 32000, chain=True, greedy="all"),
        # ordinary traffic: trees of fixed drafts, some sequences greedy
        _verify("verify_32x8_128k_some_greedy", 32, 8, 131072, greedy="some", shape=5),
        # large batch: chains of drafts that were drawn from the drafting model's probabilities
        _verify("verify_48x9_128k_sampled", 48, 9, 131072, sampled=True, chain=True),
        # an odd vocabulary, fp32 logits, ragged trees with several drawn drafts behind a node
        _verify("verify_16_ragged_50257_fp32", 16, 24, 50257, kind="fp32", sampled=True, few=3, shape=6),
        # one sequence, one stage's few layers
        _commit("commit_1x6_4_layers_int2", 1, 6, 4, cache="c2", meta="paper", shape=7),
        # a batch, all layers
        _commit("commit_48x16_32_layers", 48, 16, 32, shape=8),
        # the unquantized cache, large trees
        _commit("commit_16_ragged_24_layers_bf16", 16, 48, 24, cache="bf16", few=2, shape=9),
    ]


def _log_uniform(rng, a, b):
    return min(b, max(a, int(math.exp(rng.uniform(math.log(a), math.log(b + 1))))))


def draw(rng):
    op = rng.choices(("attn", "verify", "commit"), (50, 35, 15))[0]
    shape = rng.randrange(1 << 20)
    cache = rng.choices(("c4", "c2", "bf16"), (50, 25, 25))[0]
    meta = "paper" if cache != "bf16" and rng.random() < 0.4 else "fp16"
    nodes = _log_uniform(rng, 1, MOST_NODES)
    few = max(1, nodes // 8) if nodes > 1 and rng.random() < 0.4 else 0
    chain = rng.random() < 0.3
    while True:
        if op == "commit":
            c = _commit(None, _log_uniform(rng, 1, 64), nodes, _log_uniform(rng, 1, 40), cache, meta, few, shape)
            if sum(len(p) for p in _kept(c)) * c["layers"] <= MOST_MOVES and c["B"] * c["layers"] <= 1536:
                return c
        elif op == "verify":
            c = _verify(None, _log_uniform(rng, 1, 64), nodes, _log_uniform(rng, 1000, 151000), rng.choice(("bf16", "fp32")),
                        rng.random() < 0.5, few, chain, rng.choice(("none", "some", "all")), shape)
            if sum(_nodes(c)) * c["vocab"] <= MOST_LOGITS:
                return c
        else:
            ctx = _log_uniform(rng, 1, 131072)
            B = _log_uniform(rng, 1, 64)
            lo = max(1, ctx // 16) if B > 1 and rng.random() < 0.5 else 0
            c = _attn(None, B, ctx, nodes, rng.choice((16, 32, 64, 128)), cache, meta, lo, few, chain, shape)
            rows = [n * c["H"] for n in _nodes(c)]
            lens = _contexts(c)
            if sum(lens) <= MOST_TOKENS and sum(r * n for r, n in zip(rows, lens)) <= MOST_PAIRS:
                return c


def _contexts(case):
    if not case["lo"]:
        return [case["ctx"]] * case["B"]
    r = random.Random(case["shape"])
    return [_log_uniform(r, case["lo"], case["ctx"]) for _ in range(case["B"])]


def _nodes(case):
    """Drafted tokens of every sequence, the root among them."""
    if not case["few"]:
        return [case["nodes"]] * case["B"]
    r = random.Random(case["shape"] + 1)
    return [_log_uniform(r, case["few"], case["nodes"]) for _ in range(case["B"])]


def _parents(case):
    """Parents of every sequence's nodes: node 0 is the root, parents come before their children."""
    r = random.Random(case["shape"] + 2)
    chain = case.get("chain", False)
    return [[-1] + [i - 1 if chain else r.randrange(max(0, i - 5), i) for i in range(1, n)] for n in _nodes(case)]


def _lineage(parents, i):
    """Node i and its ancestors, the root first."""
    up = []
    while i >= 0:
        up.append(i)
        i = parents[i]
    return up[::-1]


def _kept(case):
    """The accepted nodes of every sequence of a commit case."""
    r = random.Random(case["shape"] + 3)
    return [_lineage(p, r.randrange(len(p))) for p in _parents(case)]


# ---------------------------------------------------------------------------
# Inputs, from the seed alone.

def _generator(seed, stream):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 8 + stream)
    return g


class _State:
    pass


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _starts(counts):
    return torch.cat([_int32([0]), torch.cumsum(_int32(counts), 0).to(torch.int32)])


def _pages(lens, seed):
    """Page table of sequences of these lengths, pages in random order."""
    counts = [-(-n // PAGE) for n in lens]
    ids = torch.randperm(sum(counts), generator=_generator(seed, 2), device=DEV).to(torch.int32)
    table = torch.zeros((len(lens), max(counts)), dtype=torch.int32, device=DEV)
    at = 0
    for b, k in enumerate(counts):
        table[b, :k] = ids[at:at + k]
        at += k
    return table, sum(counts)


def _regions(case):
    """Bytes per token of a page's regions (content codes, RoPE codes, metadata), and the page's size."""
    if case["cache"] == "bf16":
        return [1152], PAGE * 1152
    widths = [128 if case["cache"] == "c2" else 256, 32] + ([32] if case["meta"] == "paper" else [32, 4])
    return widths, -(-PAGE * sum(widths) // 256) * 256


def _split(cache, case):
    """Views [.., pages, tokens of a page, bytes] of the regions of packed pages [.., pages, page bytes]."""
    at, got = 0, []
    for w in _regions(case)[0]:
        got.append(cache[..., at:at + PAGE * w].unflatten(-1, (PAGE, w)))
        at += PAGE * w
    return got


def _random_cache(case, num_pages, seed):
    """Packed pages [pages, page bytes] as a writer leaves them: codes, scales around 0.15 and whole zero-points."""
    g = _generator(seed, 4)
    if case["cache"] == "bf16":
        rows = torch.randn((num_pages, PAGE * 576), generator=g, device=DEV, dtype=torch.bfloat16)
        return rows.view(torch.uint8)
    pages = torch.randint(0, 256, (num_pages, _regions(case)[1]), generator=g, device=DEV, dtype=torch.uint8)
    regions = _split(pages, case)
    scale = torch.rand((num_pages, PAGE, 9), generator=g, device=DEV) * 0.2 + 0.05
    zero = torch.randint(0, 16, (num_pages, PAGE, 9), generator=g, device=DEV)
    if case["cache"] == "c2":
        scale[..., :8] *= 4.0
        zero[..., :8] %= 4
    if case["meta"] == "paper":
        rec = regions[2]
        rec[..., :16] = scale[..., :8].bfloat16().view(torch.uint8)
        rec[..., 16:24] = zero[..., :8].to(torch.uint8)
        rec[..., 24:28] = scale[..., 8:].contiguous().view(torch.uint8)
        rec[..., 28] = zero[..., 8].to(torch.uint8)
        rec[..., 29:] = 0
    else:
        both = torch.stack([scale.half(), zero.half()], dim=-1).flatten(-2).view(torch.uint8)
        regions[2][...] = both[..., :32]
        regions[3][...] = both[..., 32:]
    return pages


def _format(case):
    from paper_2609_36760_amd import _binding as mb
    return mb.cache_format(c_bits=2 if case["cache"] == "c2" else 4, page_size=PAGE,
                           meta=mb.MLA_META_PAPER if case["meta"] == "paper" else mb.MLA_META_FP16)


def _prepare_attn(s, case, seed):
    ctx, nodes, H = _contexts(case), _nodes(case), case["H"]
    T, lens = sum(nodes), [a + b for a, b in zip(ctx, nodes)]
    s.block_table, s.num_pages = _pages(lens, seed)
    s.cache = _random_cache(case, s.num_pages, seed)
    g = _generator(seed, 0)
    s.q_lat = torch.randn((T, H, 512), generator=g, device=DEV, dtype=torch.bfloat16)
    s.q_rope = torch.randn((T, H, 64), generator=g, device=DEV, dtype=torch.bfloat16)
    s.ctx, s.cu, s.max_nodes = _int32(ctx), _starts(nodes), max(nodes)
    masks = [sum(1 << j for j in _lineage(p, i)) for p in _parents(case) for i in range(len(p))]
    s.mask = torch.tensor([m - (1 << 64) if m >> 63 else m for m in masks], dtype=torch.int64, device=DEV)
    s.out = torch.zeros((T, H, 512), dtype=torch.bfloat16, device=DEV)
    if own:         # one plan serves all layers of a step
        from paper_2609_36760_amd import _binding as mb
        from paper_2609_36760_amd import _speculate as ms
        s.split_tokens = ms.mla_tree_split_tokens(lens, s.max_nodes, H)
        s.indptr, s.num_splits, size = None, 0, 0
        if s.split_tokens:
            indptr, s.num_splits = mb.mla_plan_splits(lens, s.split_tokens)
            s.indptr = torch.from_numpy(indptr).to(DEV)
            size = ms.mla_tree_workspace_bytes(s.num_splits, s.max_nodes, H)
        s.workspace = torch.empty(size, dtype=torch.uint8, device=DEV)


def _prepare_verify(s, case, seed):
    V, nodes, parents = case["vocab"], _nodes(case), _parents(case)
    T, B = sum(nodes), len(nodes)
    g = _generator(seed, 0)
    dtype = torch.bfloat16 if case["kind"] == "bf16" else torch.float32
    s.cu, s.max_nodes = _starts(nodes), max(nodes)
    s.parents = _int32([p for q in parents for p in q])
    # a few likely tokens above a broad rest, as a language model's
    logits = torch.randn((T, V), generator=g, device=DEV) * 2.0
    peaks = torch.randint(0, V, (T, 8), generator=g, device=DEV)
    logits.scatter_add_(1, peaks, 10.0 + 2.0 * torch.randn((T, 8), generator=g, device=DEV))
    s.logits = logits.to(dtype)
    # the drafting model is near the target
    logits += 0.7 * torch.randn((T, V), generator=g, device=DEV)
    first = torch.repeat_interleave(s.cu[:-1], _int32(nodes))
    above = (first + s.parents.clamp(min=0)).long()         # row of every node's parent
    if case["sampled"]:
        s.probs = torch.softmax(logits, dim=1)
        noise = torch.empty((T, V), device=DEV).exponential_(generator=g)
        s.tokens = (torch.log(s.probs[above]) - torch.log(noise)).argmax(1).to(torch.int32)
    else:
        s.probs = None
        likely = logits.topk(min(V, 8), dim=1).indices
        rank = _int32([sum(1 for j in range(1, i) if q[j] == q[i]) for q in parents for i in range(len(q))]).long()
        s.tokens = likely[above, rank.clamp(max=likely.shape[1] - 1)].to(torch.int32)
    every = {"none": 0, "some": 4, "all": 1}[case["greedy"]]
    s.temperature = torch.tensor([0.0 if every and b % every == 0 else 0.6 + 0.1 * (b % 6) for b in range(B)], device=DEV)
    s.u_accept = torch.rand((T,), generator=g, device=DEV)
    s.u_draw = torch.rand((B,), generator=g, device=DEV)
    s.path = torch.empty((B, s.max_nodes), dtype=torch.int32, device=DEV)
    s.emitted = torch.empty((B, s.max_nodes), dtype=torch.int32, device=DEV)
    s.logprobs = torch.empty((B, s.max_nodes), dtype=torch.float32, device=DEV)
    s.keep = torch.empty((B,), dtype=torch.int32, device=DEV)
    if own:
        from paper_2609_36760_amd import _speculate as ms
        s.workspace = torch.empty(ms.mla_verify_workspace_bytes(T, B, V), dtype=torch.uint8, device=DEV)


def _prepare_commit(s, case, seed):
    kept, nodes = _kept(case), _nodes(case)
    r = random.Random(case["shape"] + 4)
    ctx = [r.randrange(1, 200) for _ in nodes]
    s.block_table, s.num_pages = _pages([a + b for a, b in zip(ctx, nodes)], seed)
    size = _regions(case)[1]
    s.caches = torch.randint(0, 256, (case["layers"], s.num_pages, size), generator=_generator(seed, 4), device=DEV, dtype=torch.uint8)
    s.max_nodes = max(nodes)
    s.path = _int32([p + [-1] * (s.max_nodes - len(p)) for p in kept])
    s.keep = _int32([len(p) for p in kept])
    s.ctx = _int32(ctx)
    s.lens = torch.empty_like(s.ctx)
    if own:         # the table of a model's layers is made once
        from paper_2609_36760_amd import _speculate as ms
        s.layers = ms.layer_caches(list(s.caches))


def prepare(case, seed):
    s = _State()
    s.case = case
    {"attn": _prepare_attn, "verify": _prepare_verify, "commit": _prepare_commit}[case["op"]](s, case, seed)
    return s


# ---------------------------------------------------------------------------
# The library's calls.

def _run_own(s):
    from paper_2609_36760_amd import _speculate as ms
    case = s.case
    if case["op"] == "attn":
        call = ms.mla_bf16_tree_attn if case["cache"] == "bf16" else ms.mla_lowbit_tree_attn
        call(_format(case), s.q_lat, s.q_rope, s.cache, s.num_pages, s.block_table, s.ctx, s.cu, s.mask, s.max_nodes,
             TAU, s.out, split_tokens=s.split_tokens, split_indptr=s.indptr, num_splits=s.num_splits, workspace=s.workspace)
        return {"out": s.out}
    if case["op"] == "verify":
        ms.mla_verify_tree(s.logits, s.tokens, s.parents, s.cu, s.max_nodes, s.u_accept, s.u_draw, s.path, s.emitted,
                           s.keep, s.workspace, temperature=s.temperature, draft_probs=s.probs, logprobs=s.logprobs)
        return {"path": s.path, "tokens": s.emitted, "keep": s.keep, "logprobs": s.logprobs}
    call = ms.mla_bf16_commit if case["cache"] == "bf16" else ms.mla_lowbit_commit
    call(_format(case), s.layers, s.num_pages, s.block_table, s.ctx, s.path, s.keep, s.lens)
    return {"caches": s.caches, "lens": s.lens}


# ---------------------------------------------------------------------------
# The plain forms.

def _codes(raw, bits):
    """Channel 2i of a word at bits [bits i, bits (i+1)), channel 2i + 1 in the same bits of its upper half."""
    half = raw.contiguous().view(torch.int16).int().unflatten(-1, (-1, 2)) & 0xFFFF
    shift = torch.arange(0, 16, bits, device=DEV, dtype=torch.int32)
    return ((half[..., None, :] >> shift[:, None]) & ((1 << bits) - 1)).flatten(-3)


def _plain_rows(s, seqs, n):
    """The first ``n`` cached tokens of sequences ``seqs`` as fp32 [sequences, n, 576]."""
    case = s.case
    t = torch.arange(n, device=DEV)
    page, off = s.block_table[seqs][:, t // PAGE].long(), t % PAGE
    parts = [r[page, off[None]] for r in _split(s.cache, case)]
    if case["cache"] == "bf16":
        return parts[0].contiguous().view(torch.bfloat16).float()
    bits = 2 if case["cache"] == "c2" else 4
    code = torch.cat([_codes(parts[0], bits), _codes(parts[1], 4)], dim=-1).float().unflatten(-1, (9, 64))
    if case["meta"] == "paper":
        rec = parts[2]
        scale = torch.cat([rec[..., :16].contiguous().view(torch.bfloat16).float(),
                           rec[..., 24:28].contiguous().view(torch.float32)], dim=-1)
        zero = torch.cat([rec[..., 16:24], rec[..., 28:29]], dim=-1).float()
    else:
        both = torch.cat([parts[2], parts[3]], dim=-1).view(torch.float16).float().unflatten(-1, (9, 2))
        scale, zero = both[..., 0], both[..., 1]
    return (scale[..., None] * (code - zero[..., None])).flatten(-2)


def _plain_attn(s):
    """Sequences of one length and one number of nodes together."""
    case = s.case
    H, ctx, nodes = case["H"], _contexts(case), _nodes(case)
    alike = {}
    for b, key in enumerate(zip(ctx, nodes)):
        alike.setdefault(key, []).append(b)
    for (c, n), seqs in alike.items():
        seqs = torch.tensor(seqs, device=DEV)
        rows = s.cu[seqs].long()[:, None] + torch.arange(n, device=DEV)
        x = _plain_rows(s, seqs, c + n)
        q = torch.cat([s.q_lat[rows], s.q_rope[rows]], dim=-1).float().flatten(1, 2)
        z = torch.matmul(q, x.transpose(1, 2).contiguous()).mul_(TAU)
        hidden = ((s.mask[rows][..., None] >> torch.arange(n, device=DEV)) & 1) == 0
        z[..., c:].masked_fill_(hidden.repeat_interleave(H, dim=1), -math.inf)
        p = z.sub_(z.amax(-1, keepdim=True)).exp_()
        y = torch.matmul(p, x[..., :512].contiguous()) / p.sum(-1, keepdim=True)
        s.out[rows] = y.unflatten(1, (n, H)).bfloat16()
    return {"out": s.out}


def _plain_verify(s):
    """All sequences together, a level of the trees after the other, its children one after the other."""
    case, V = s.case, s.case["vocab"]
    parents = _parents(case)
    B = len(parents)
    levels = max(len(_lineage(p, i)) for p in parents for i in range(len(p)))
    width = max(sum(1 for a in p[1:] if a == v) for p in parents for v in range(len(p)))
    # children of every node in their order, -1: none
    table = [[[i for i in range(1, len(p)) if p[i] == v] for v in range(len(p))] for p in parents]
    child = _int32([c + [-1] * (max(1, width) - len(c)) for p in table for c in p])
    seq = torch.arange(B, device=DEV)
    first = s.cu[:-1].long()
    s.path.fill_(-1)
    s.emitted.fill_(-1)
    s.logprobs.zero_()
    s.keep.fill_(1)
    s.path[:, 0] = 0
    at = torch.zeros(B, dtype=torch.long, device=DEV)
    walking = torch.ones(B, dtype=torch.bool, device=DEV)
    greedy = s.temperature == 0
    heat = torch.where(greedy, torch.ones_like(s.temperature), s.temperature).double()[:, None]
    for _ in range(levels):
        row = first + at
        l = s.logits[row].double() / heat
        best = s.logits[row].float().argmax(1)
        p = torch.softmax(l, dim=1)
        p = torch.where(greedy[:, None], torch.zeros_like(p).scatter_(1, best[:, None], 1.0), p)
        r = p.clone()
        took = torch.zeros_like(walking)
        for k in range(width):
            node = child[row, k].long()
            here = walking & ~took & (node >= 0)
            c = first + node.clamp(min=0)
            x = s.tokens[c].long()[:, None]
            mass = r.gather(1, x)[:, 0]
            if case["sampled"]:
                q = s.probs[row].double()
                chance = s.u_accept[c].double() * torch.where(greedy, r.sum(1), q.gather(1, x)[:, 0])
                left = (r - q).clamp(min=0.0)
                left = left / left.sum(1, keepdim=True)
            else:
                chance = s.u_accept[c].double() * r.sum(1)
            yes = here & torch.where(greedy, mass > 0, chance < mass)
            no = here & ~yes & ~greedy
            if case["sampled"]:
                r = torch.where((no & torch.isfinite(left[:, 0]))[:, None], left, r)
            else:
                r = torch.where(no[:, None], r.scatter(1, x, 0.0), r)
            b = seq[yes]
            s.path[b, s.keep[b].long()] = node[yes].to(torch.int32)
            s.emitted[b, s.keep[b].long() - 1] = x[yes, 0].to(torch.int32)
            s.logprobs[b, s.keep[b].long() - 1] = torch.log(p[yes].gather(1, x[yes]))[:, 0].float()
            s.keep[b] += 1
            at[b] = node[yes]
            took = took | yes
        cum = torch.cumsum(r, dim=1)
        x = (cum > s.u_draw.double()[:, None] * cum[:, -1:]).to(torch.uint8).argmax(1)
        end = walking & ~took
        b = seq[end]
        s.emitted[b, s.keep[b].long() - 1] = x[end].to(torch.int32)
        s.logprobs[b, s.keep[b].long() - 1] = torch.log(p[end].gather(1, x[end][:, None]))[:, 0].float()
        walking = took
    return {"path": s.path, "tokens": s.emitted, "keep": s.keep, "logprobs": s.logprobs}


def _plain_commit(s):
    k = torch.arange(s.max_nodes, device=DEV)
    here = k < s.keep[:, None]
    seq = torch.arange(s.ctx.shape[0], device=DEV)[:, None].expand_as(here)[here]
    src, dst = (s.ctx[:, None] + s.path)[here].long(), (s.ctx[:, None] + k)[here].long()
    sp, dp = s.block_table[seq, src // PAGE].long(), s.block_table[seq, dst // PAGE].long()
    for r in _split(s.caches, s.case):
        r[:, dp, dst % PAGE] = r[:, sp, src % PAGE]
    torch.add(s.ctx, s.keep, out=s.lens)
    return {"caches": s.caches, "lens": s.lens}


def run(s):
    if own:
        return _run_own(s)
    return {"attn": _plain_attn, "verify": _plain_verify, "commit": _plain_commit}[s.case["op"]](s)


# ---------------------------------------------------------------------------

def work(case):
    nodes = _nodes(case)
    T = sum(nodes)
    if case["op"] == "attn":
        H, ctx = case["H"], _contexts(case)
        pairs = sum(c * n for c, n in zip(ctx, nodes))
        pairs += sum(len(_lineage(p, i)) for p in _parents(case) for i in range(len(p)))
        cached = (sum(ctx) + T) * sum(_regions(case)[0])
        return {"bytes": cached + T * (H * (1152 + 1024) + 8), "flops": 2176 * pairs * H}
    if case["op"] == "verify":
        per = 2 if case["kind"] == "bf16" else 4
        B, V = case["B"], case["vocab"]
        # every row's logits (which ones the walk meets is not known before), and one row of probabilities a sequence
        return {"bytes": T * V * per + (B * V * 4 if case["sampled"] else 0) + T * 12 + B * 16, "flops": T * V * 4}
    moved = sum(1 for p in _kept(case) for k, i in enumerate(p) if i != k)
    return {"bytes": 2 * moved * case["layers"] * sum(_regions(case)[0]) + case["B"] * (12 + 4 * max(nodes)), "flops": 0}


# ---------------------------------------------------------------------------
# The same in 64 bits, from the definitions.

def _exact_attn(case, s):
    """Sequence by sequence, channel by channel from the code words; every node with its own list of keys."""
    H, widths = case["H"], _regions(case)[0]
    out = torch.zeros((s.q_lat.shape[0], H, 512), dtype=torch.float64, device=DEV)
    flat = s.cache.reshape(s.num_pages, -1)
    a = 0
    for b, (c, parents) in enumerate(zip(_contexts(case), _parents(case))):
        pos = torch.arange(c + len(parents), device=DEV)
        page, off = torch.index_select(s.block_table[b], 0, pos // PAGE).long(), pos % PAGE

        def region(k):
            base = PAGE * sum(widths[:k]) + off * widths[k]
            return flat[page[:, None], base[:, None] + torch.arange(widths[k], device=DEV)]

        if case["cache"] == "bf16":
            x = region(0).contiguous().view(torch.bfloat16).double()
        else:
            def value(k, channels, bits):
                per = 32 // bits
                ch = torch.arange(channels, device=DEV)
                bit = (ch // per) * 32 + 16 * (ch % 2) + bits * ((ch % per) // 2)
                return (torch.index_select(region(k), 1, bit // 8).int() >> (bit % 8)) & (2 ** bits - 1)

            meta = region(2)
            if case["meta"] == "paper":
                sc, sr = meta[:, :16].contiguous().view(torch.bfloat16), meta[:, 24:28].contiguous().view(torch.float32)
                zc, zr = meta[:, 16:24], meta[:, 28:29]
            else:
                mc, mr = meta.contiguous().view(torch.half), region(3).contiguous().view(torch.half)
                sc, zc, sr, zr = mc[:, 0::2], mc[:, 1::2], mr[:, :1], mr[:, 1:]
            group = torch.arange(512, device=DEV) // 64
            xc = (value(0, 512, 2 if case["cache"] == "c2" else 4).double() - zc.double()[:, group]) * sc.double()[:, group]
            x = torch.cat([xc, (value(1, 64, 4).double() - zr.double()) * sr.double()], 1)
        xt = x.T.contiguous()
        for i in range(len(parents)):
            q = torch.cat([s.q_lat[a + i], s.q_rope[a + i]], 1).double()
            z = torch.matmul(q, xt) / math.sqrt(192.0)
            seen = torch.zeros(len(pos), dtype=torch.bool, device=DEV)
            seen[:c] = True
            seen[[c + j for j in _lineage(parents, i)]] = True
            w = torch.where(seen, z, -math.inf)
            out[a + i] = torch.matmul(torch.exp(w - torch.logsumexp(w, 1, keepdim=True)), x[:, :512].contiguous())
        a += len(parents)
    return {"out": out}


def _exact_verify(case, s):
    """One sequence after the other on the host's terms, with logarithms; only what the walk meets."""
    cu, u, ud = s.cu.tolist(), s.u_accept.tolist(), s.u_draw.tolist()
    tokens, heat = s.tokens.tolist(), s.temperature.tolist()
    got = {k: torch.full((len(cu) - 1, s.max_nodes), v, dtype=t) for k, v, t in
           (("path", -1, torch.int32), ("tokens", -1, torch.int32), ("logprobs", 0.0, torch.float64))}
    keep = []
    for b, parents in enumerate(_parents(case)):
        base, v, path = cu[b], 0, [0]
        while True:
            l = s.logits[base + v].double()
            if heat[b] == 0.0:
                best = int((l == l.max()).nonzero()[0, 0])
                logp = torch.full_like(l, -math.inf)
                logp[best] = 0.0
            else:
                logp = l / torch.tensor(heat[b], dtype=torch.float32).double().item()
                logp = logp - torch.logsumexp(logp, 0)
            r, taken = torch.exp(logp), None
            for i in (i for i in range(1, len(parents)) if parents[i] == v):
                x = tokens[base + i]
                mass = r[x].item()
                if heat[b] == 0.0:
                    yes = mass > 0
                elif case["sampled"]:
                    q = s.probs[base + v].double()
                    yes = u[base + i] * q[x].item() < mass
                    if not yes:
                        left = torch.where(r > q, r - q, 0.0)
                        r = left / left.sum() if left.sum().item() > 0 else r
                else:
                    yes = u[base + i] * r.sum().item() < mass
                    if not yes:
                        r[x] = 0.0
                if yes:
                    taken = i
                    break
            if taken is None:
                up = torch.cumsum(r, 0)
                x = int(torch.searchsorted(up, torch.tensor([ud[b]], device=DEV, dtype=torch.float64) * up[-1], right=True))
            got["tokens"][b, len(path) - 1] = x
            got["logprobs"][b, len(path) - 1] = logp[x].item()
            if taken is None:
                break
            path.append(taken)
            v = taken
        got["path"][b, :len(path)] = torch.tensor(path, dtype=torch.int32)
        keep.append(len(path))
    return {"path": got["path"], "tokens": got["tokens"], "keep": torch.tensor(keep, dtype=torch.int32), "logprobs": got["logprobs"]}


def exact(case, seed):
    if case["op"] == "commit":      # bytes that move, no computed numbers
        return None
    s = prepare(case, seed)
    return _exact_attn(case, s) if case["op"] == "attn" else _exact_verify(case, s)
