"""The prompt-side operators, in their plain form and as the library's calls.

A program that serves a latent-attention layer runs them around the decode:

* ``append``: a prompt's (or a step's) latents are normalized, their RoPE keys
  rotated, both quantized into the paged cache and handed on as dense rows; the
  tokens are then read back from the cache as a later chunk reads its prefix;
* ``gather``: the cached tokens of a batch are read back as dense rows;
* ``rope``: the queries' RoPE channels are rotated;
* ``attn``: attention in its expanded form, 128 + 64 channels a key (the 64
  shared by all heads) and 128 a value: prompts, prompt chunks behind a
  prefix, single tokens, and a prefix by itself, which some rows lack.

Heads per GPU 16, 32, 64 and 128 (a 128-head layer under tensor parallelism of
8, 4, 2 and 1), 64-token pages in random order, INT4 and INT2 content, both
metadata formats, with and without BF16 protection, and the BF16 cache.

Sizes and lengths are part of a case and do not depend on the seed.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda"
PAGE, SINK, RECENT = 64, 4, 128
TAU = 1.0 / math.sqrt(192.0)
EPS = 1e-6
MOST_PAIRS = 1 << 33            # (row, key, head) scores of an attention case, hidden ones included
MOST_SEEN = MOST_PAIRS // 2     # without the hidden ones
MOST_VECTORS = 1 << 23          # (key, head) pairs of an attention case
MOST_TOKENS = {"append": 1 << 16, "gather": 1 << 17}


def _attn(name, B, ctx, H, q=0, causal=True, lo=0, gaps=False, lens_seed=0):
    """``ctx``: prompt or prefix tokens of every sequence (with ``lo`` the upper
    end of log-uniform lengths); ``q``: new rows behind the prefix, 0: the prompt
    itself; ``gaps``: every fourth sequence has no prefix."""
    c = dict(op="attn", B=B, ctx=ctx, lo=lo, lens_seed=lens_seed, H=H, q=q, causal=causal, gaps=gaps)
    return dict(c, name=name) if name else c


def _cached(name, op, B, n, base=0, cache="c4", meta="fp16", prot=False, weight=False, halves=False, lo=0, lens_seed=0):
    """``n`` tokens of each sequence (``lo``: ragged) behind ``base`` older ones."""
    c = dict(op=op, B=B, n=n, lo=lo, lens_seed=lens_seed, base=base, cache=cache, meta=meta, prot=prot)
    if op == "append":
        c.update(weight=weight, halves=halves)
    return dict(c, name=name) if name else c


def _rope(name, n, H, halves=False):
    c = dict(op="rope", n=n, H=H, halves=halves)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the smallest call: one short chat prompt on one GPU of eight
        _attn("attn_h16_prompt_1x64", 1, 64, 16),
        # ordinary traffic: a batch of prompts of unequal, odd lengths
        _attn("attn_h128_prompts_12_ragged", 12, 2047, 128, lo=65, lens_seed=5),
        # one long prompt, all heads
        _attn("attn_h128_prompt_1x8k", 1, 8192, 128),
        # chunked prefill: the next rows of a long document behind its prefix, on one GPU of eight
        _attn("attn_h16_chunk_500_on_32k", 1, 32268, 16, q=500),
        # single tokens of a running batch over expanded keys
        _attn("attn_h32_tokens_24x2k", 24, 3000, 32, q=1, lo=1000, lens_seed=6),
        # the prefix part of a chunk by itself, which new requests lack
        _attn("attn_h64_prefix_8x129_ragged", 8, 4100, 64, q=129, causal=False, lo=300, gaps=True, lens_seed=7),
        # a prefill chunk of eight prompts into the INT4 cache under protection
        _cached("append_8x8k_prot", "append", 8, 8192, prot=True),
        # a decode step's tokens into the INT2 cache, in the paper's storage, with a norm weight
        _cached("append_64x1_int2_paper", "append", 64, 1, base=700, cache="c2", meta="paper", weight=True, halves=True),
        # the prefix of a long document, and of a ragged batch in the paper's storage under protection
        _cached("gather_1x128k", "gather", 1, 131072),
        _cached("gather_16_ragged_paper_prot", "gather", 16, 1500, lo=100, lens_seed=8, meta="paper", prot=True),
        # the queries of a short prompt on one GPU of eight, and of an 8K prompt with all heads
        _rope("rope_h16_77", 77, 16, halves=True),
        _rope("rope_h128_8k", 8192, 128),
    ]


def _log_uniform(rng, a, b):
    return min(b, max(a, int(math.exp(rng.uniform(math.log(a), math.log(b + 1))))))


def draw(rng):
    op = rng.choices(("attn", "append", "gather", "rope"), (50, 20, 15, 15))[0]
    seed = rng.randrange(1 << 20)
    if op == "rope":
        return _rope(None, _log_uniform(rng, 1, 8192), rng.choice((16, 32, 64, 128)), rng.random() < 0.5)
    if op != "attn":
        cache = rng.choices(("c4", "c2", "bf16"), (50, 25, 25))[0]
        meta = "paper" if cache != "bf16" and rng.random() < 0.4 else "fp16"
        prot = cache != "bf16" and rng.random() < 0.4
        total = _log_uniform(rng, 1, MOST_TOKENS[op])
        B = min(total, _log_uniform(rng, 1, 64))
        n = max(1, total // B)
        lo = max(1, n // 16) if rng.random() < 0.5 and n > 1 else 0
        base = rng.choice((0, 0, rng.randrange(1, 500)))
        return _cached(None, op, B, n, base, cache, meta, prot, rng.random() < 0.5, rng.random() < 0.5, lo, seed)
    H = rng.choice((16, 32, 64, 128))
    kind = rng.choice(("prompt", "chunk", "token", "prefix"))
    q = {"prompt": 0, "chunk": _log_uniform(rng, 2, 2048), "token": 1, "prefix": _log_uniform(rng, 1, 512)}[kind]
    while True:
        ctx = _log_uniform(rng, 1, 8192 if kind == "prompt" else 32768)
        B = _log_uniform(rng, 1, 32)
        lo = max(1, ctx // 16) if B > 1 and rng.random() < 0.6 else 0
        c = _attn(None, B, ctx, H, q, kind != "prefix", lo, kind == "prefix" and B > 3, seed)
        ql, kl = _attn_lens(c)
        pairs = H * sum(a * b for a, b in zip(ql, kl))
        if H * sum(kl) <= MOST_VECTORS and pairs <= MOST_PAIRS and work(c)["flops"] <= 640 * MOST_SEEN:
            return c


def _ragged(case, top):
    if not case["lo"]:
        return [top] * case["B"]
    r = random.Random(case["lens_seed"])
    return [_log_uniform(r, case["lo"], top) for _ in range(case["B"])]


def _attn_lens(case):
    """Query rows and keys of every sequence."""
    ctx, q = _ragged(case, case["ctx"]), case["q"]
    if case["gaps"]:
        ctx = [0 if b % 4 == 1 else n for b, n in enumerate(ctx)]
    if not q:
        return ctx, ctx
    return [q] * len(ctx), [n + q if case["causal"] else n for n in ctx]


# ---------------------------------------------------------------------------
# Inputs, from the seed alone.

def _generator(seed, stream):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 8 + stream)
    return g


class _State:
    pass


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.bfloat16)


def _rotation_table(positions):
    """fp32 [positions, 64]: cosines, then sines, of position * 10000^(-2i/64)."""
    theta = 10000.0 ** (-torch.arange(32, device=DEV, dtype=torch.float64) / 32.0)
    a = torch.arange(positions, device=DEV, dtype=torch.float64)[:, None] * theta
    return torch.cat([a.cos(), a.sin()], dim=1).float()


def _attn_inputs(case, seed):
    """Queries [Tq, H, 192], expanded keys and values [Tk, H, 256] as one product leaves them (128 | 128), RoPE keys."""
    ql, kl = _attn_lens(case)
    g = _generator(seed, 0)
    q, kv, kr = _normal(g, sum(ql), case["H"], 192), _normal(g, sum(kl), case["H"], 256), _normal(g, sum(kl), 64)
    # scores with a spread of about 2, a few channels standing out
    gain = torch.ones(192, device=DEV, dtype=torch.bfloat16)
    gain[torch.randperm(128, generator=g, device=DEV)[:4]] = 4.0
    return q * gain, kv, kr


def _pages(case, lens, seed):
    """Page table of sequences of these lengths, pages in random order."""
    counts = [-(-n // PAGE) for n in lens]
    ids = torch.randperm(sum(counts), generator=_generator(seed, 2), device=DEV).to(torch.int32)
    table = torch.zeros((len(lens), max(counts)), dtype=torch.int32, device=DEV)
    at = 0
    for b, k in enumerate(counts):
        table[b, :k] = ids[at:at + k]
        at += k
    return table, sum(counts)


def _page_layout(case):
    """Byte offsets of a page's regions (content codes, RoPE codes, metadata) and its size."""
    cc = 512 * (2 if case["cache"] == "c2" else 4) // 8
    at = [0, PAGE * cc, PAGE * (cc + 32), PAGE * (cc + 64)]
    end = at[2] + PAGE * (32 if case["meta"] == "paper" else 36)
    return cc, at, -(-end // 256) * 256


def _random_cache(case, num_pages, seed):
    """Packed pages as a writer leaves them: codes, scales around 0.3 and whole zero-points."""
    g = _generator(seed, 4)
    if case["cache"] == "bf16":
        return _normal(g, num_pages, PAGE * 576).view(torch.uint8).reshape(-1)
    cc, at, size = _page_layout(case)
    pages = torch.randint(0, 256, (num_pages, size), generator=g, device=DEV, dtype=torch.uint8)
    top = 4 if case["cache"] == "c2" else 16
    scale = torch.rand((num_pages, PAGE, 9), generator=g, device=DEV) * 0.4 + 0.1
    zero = torch.randint(0, 16, (num_pages, PAGE, 9), generator=g, device=DEV)
    zero[..., :8] %= top
    if case["meta"] == "paper":
        rec = torch.zeros((num_pages, PAGE, 32), dtype=torch.uint8, device=DEV)
        rec[..., :16] = scale[..., :8].bfloat16().view(torch.uint8)
        rec[..., 16:24] = zero[..., :8].to(torch.uint8)
        rec[..., 24:28] = scale[..., 8:].contiguous().view(torch.uint8)
        rec[..., 28] = zero[..., 8].to(torch.uint8)
        pages[:, at[2]:at[2] + PAGE * 32] = rec.reshape(num_pages, -1)
    else:
        both = torch.stack([scale.half(), zero.half()], dim=-1)
        for part, where in ((both[:, :, :8], at[2]), (both[:, :, 8:], at[3])):
            raw = part.contiguous().view(torch.uint8).reshape(num_pages, -1)
            pages[:, where:where + raw.shape[1]] = raw
    return pages.reshape(-1)


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _format(case):
    from paper_2609_36760_amd import _binding as mb
    return mb.cache_format(c_bits=2 if case["cache"] == "c2" else 4, page_size=PAGE,
                           meta=mb.MLA_META_PAPER if case["meta"] == "paper" else mb.MLA_META_FP16)


def _tokens(case, n, seed):
    """Latents before their norm, keys before their rotation, and the norm's weight."""
    g = _generator(seed, 1)
    gain = torch.ones(512, device=DEV)
    gain[torch.randperm(512, generator=g, device=DEV)[:5]] = 10.0
    x = (torch.randn((n, 512), generator=g, device=DEV) * gain * 3.0).bfloat16()
    i = torch.arange(64, device=DEV) // 2
    k = (torch.randn((n, 64), generator=g, device=DEV) * (0.1 * 50.0 ** (i / 31.0))).bfloat16()
    w = (1.0 + 0.2 * torch.randn(512, generator=g, device=DEV)).bfloat16() if case["weight"] else None
    return x, k, w


def prepare(case, seed):
    s = _State()
    s.case = case
    op = case["op"]
    if op == "rope":
        g = _generator(seed, 0)
        s.q = _normal(g, case["n"], case["H"], 192)
        s.positions = torch.randint(0, 8192, (case["n"],), generator=g, device=DEV).to(torch.int32)
        s.table = _rotation_table(8192)
        s.out = torch.empty((case["n"], case["H"], 64), dtype=torch.bfloat16, device=DEV)
        return s
    if op == "attn":
        ql, kl = _attn_lens(case)
        s.q, s.kv, s.kr = _attn_inputs(case, seed)
        s.out = torch.zeros((sum(ql), case["H"], 128), dtype=torch.bfloat16, device=DEV)
        s.lse = torch.zeros((sum(ql), case["H"]), dtype=torch.float32, device=DEV)
        if own:         # one plan serves all layers of a step
            from paper_2609_36760_amd import _prefill as mp
            plan, s.info = mp.mla_plan_prefill(ql, kl, case["H"], case["causal"])
            s.plan = torch.from_numpy(plan).to(DEV)
            s.workspace = torch.empty(s.info.workspace_bytes, dtype=torch.uint8, device=DEV)
        return s
    new = _ragged(case, case["n"])
    lens = [case["base"] + n for n in new]
    T = sum(new)
    s.block_table, s.num_pages = _pages(case, lens, seed)
    s.lens, s.first = _int32(lens), _int32([case["base"]] * len(new))
    s.cu = torch.cat([_int32([0]), torch.cumsum(_int32(new), 0).to(torch.int32)])
    s.seq = torch.repeat_interleave(torch.arange(len(new), device=DEV, dtype=torch.int32), _int32(new))
    s.pos = (torch.arange(T, device=DEV, dtype=torch.int32) - s.cu[s.seq.long()] + case["base"])
    s.slots = s.block_table[s.seq.long(), (s.pos // PAGE).long()].long() * PAGE + s.pos % PAGE
    s.prot_slot = torch.randperm(len(new), generator=_generator(seed, 3), device=DEV).to(torch.int32)
    s.prot = _normal(_generator(seed, 5), len(new) * (SINK + RECENT), 576) if case["prot"] else None
    s.c_out = torch.empty((T, 512), dtype=torch.bfloat16, device=DEV)
    s.k_out = torch.empty((T, 64), dtype=torch.bfloat16, device=DEV)
    if op == "append":
        s.x, s.k, s.w = _tokens(case, T, seed)
        s.rotary = _rotation_table(max(lens))
        s.c_new, s.k_new = torch.empty_like(s.c_out), torch.empty_like(s.k_out)
        size = PAGE * 1152 if case["cache"] == "bf16" else _page_layout(case)[2]
        s.cache = torch.zeros(s.num_pages * size, dtype=torch.uint8, device=DEV)
    else:
        s.cache = _random_cache(case, s.num_pages, seed)
    return s


# ---------------------------------------------------------------------------
# The library's calls.

def _run_own(s):
    from paper_2609_36760_amd import _binding as mb
    from paper_2609_36760_amd import _prefill as mp
    case = s.case
    if case["op"] == "attn":
        mp.mla_prefill_attn(s.info, s.plan, s.q[..., :128], s.q[..., 128:], s.kv[..., :128], s.kr, s.kv[..., 128:],
                            TAU, s.out, s.lse, s.workspace)
        return {"out": s.out, "lse": s.lse}
    if case["op"] == "rope":
        rot = mp.rotation(s.table, mp.MLA_ROPE_HALVES if case["halves"] else mp.MLA_ROPE_PAIRS)
        mp.mla_rope_queries(rot, s.q[..., 128:], s.positions, s.out)
        return {"out": s.out}
    fmt, bf16, prot = _format(case), case["cache"] == "bf16", case["prot"]
    policy = mb.protect_policy(SINK, RECENT) if prot else None
    out = {}
    if case["op"] == "append":
        rot = mp.rotation(s.rotary, mp.MLA_ROPE_HALVES if case["halves"] else mp.MLA_ROPE_PAIRS)
        norm = mp.rms_norm(EPS, s.w)
        if prot:
            mp.mla_lowbit_norm_rope_append_protected(fmt, policy, norm, rot, s.x, s.k, s.pos, s.slots, s.cache,
                                                     s.num_pages, s.seq, s.lens, s.prot_slot, s.prot, case["B"],
                                                     s.c_new, s.k_new)
        else:
            call = mp.mla_bf16_norm_rope_append if bf16 else mp.mla_lowbit_norm_rope_append
            call(fmt, norm, rot, s.x, s.k, s.pos, s.slots, s.cache, s.num_pages, s.c_new, s.k_new)
        out = {"c_new": s.c_new, "k_new": s.k_new}
        if prot:
            out["prot"] = s.prot
    if prot:
        mp.mla_lowbit_gather_protected(fmt, policy, s.cache, s.num_pages, s.block_table, s.cu, s.lens, s.prot, case["B"],
                                       s.prot_slot, s.c_out, s.k_out, s.first)
    else:
        call = mp.mla_bf16_gather if bf16 else mp.mla_lowbit_gather
        call(fmt, s.cache, s.num_pages, s.block_table, s.cu, s.c_out, s.k_out, s.first)
    return dict(out, c=s.c_out, k=s.k_out)


# ---------------------------------------------------------------------------
# The plain forms.

def _plain_attn(s):
    case = s.case
    H, scale = case["H"], TAU
    outs, lses, a, e = [], [], 0, 0
    for nq, nk in zip(*_attn_lens(case)):
        step = max(1, min(H, (1 << 32) // max(1, nq * nk)))
        o = torch.empty((nq, H, 128), dtype=torch.bfloat16, device=DEV)
        l = torch.empty((nq, H), dtype=torch.float32, device=DEV)
        hidden = None
        if case["causal"]:
            i, j = torch.arange(nq, device=DEV), torch.arange(nk, device=DEV)
            hidden = j[None, :] > i[:, None] + (nk - nq)
        for h in range(0, H, step):
            q = s.q[a:a + nq, h:h + step].float().transpose(0, 1)
            kv = s.kv[e:e + nk, h:h + step].float().transpose(0, 1)
            k = torch.cat([kv[..., :128], s.kr[e:e + nk].float().expand(q.shape[0], nk, 64)], dim=-1)
            z = torch.matmul(q.contiguous(), k.transpose(1, 2).contiguous()) * scale
            if hidden is not None:
                z.masked_fill_(hidden, -math.inf)
            if nk:
                top = z.amax(-1, keepdim=True)
                top = torch.where(top == -math.inf, torch.zeros_like(top), top)
            else:
                top = torch.zeros((q.shape[0], nq, 1), device=DEV)
            p = torch.exp(z.sub_(top))
            total = p.sum(-1, keepdim=True)
            y = torch.matmul(p, kv[..., 128:].contiguous()) / torch.where(total == 0, torch.ones_like(total), total)
            o[:, h:h + step] = y.transpose(0, 1).bfloat16()
            l[:, h:h + step] = (top + torch.log(total))[..., 0].transpose(0, 1)
        outs.append(o)
        lses.append(l)
        a, e = a + nq, e + nk
    return {"out": torch.cat(outs), "lse": torch.cat(lses)}


def _plain_rotate(x, rows, halves):
    """Rotated channels (last axis) by the table rows, in 64 bits: the codes behind them step at borders."""
    cos, sin = rows[..., :32].double(), rows[..., 32:].double()
    x = x.double()
    if halves:
        a, b = x[..., :32], x[..., 32:]
        return torch.cat([a * cos - b * sin, a * sin + b * cos], dim=-1).float().bfloat16()
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack([a * cos - b * sin, a * sin + b * cos], dim=-1).flatten(-2).float().bfloat16()


def _plain_norm(x, w):
    x = x.double()
    r = 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + _eps())
    return ((x if w is None else x * w.double()) * r).float().bfloat16()


def _eps():
    """The fp32 value that a caller's 1e-6 becomes."""
    return torch.tensor(EPS, dtype=torch.float32).item()


def _plain_quantized(x, bits, scale_type):
    """bf16 values that a cache of ``bits``-bit codes holds for rows ``x``, groups of 64 channels.  The two quotients
    are fp32 ones, correctly rounded (taken from 64 bits: codes step at borders)."""
    m = float((1 << bits) - 1)
    g = x.float().reshape(x.shape[0], -1, 64)
    low, high = g.amin(-1, keepdim=True), g.amax(-1, keepdim=True)
    s = ((high - low).clamp(min=1e-8).double() / m).float()
    z = torch.round((-low.double() / s.double()).float()).clamp(0.0, m)
    code = torch.round((g.double() / s.double()).float() + z).clamp(0.0, m)
    return (s.to(scale_type).float() * (code - z)).reshape(x.shape).bfloat16()


def _plain_protected(s):
    """Whether each token is protected, and its row in the protection buffers."""
    pos, L = s.pos.long(), s.lens[s.seq.long()].long()
    kept = (pos < SINK) | (pos >= L - RECENT)
    row = torch.where(pos < SINK, pos, SINK + (pos - SINK) % RECENT)
    return kept, s.prot_slot[s.seq.long()].long() * (SINK + RECENT) + row


def _plain_read(s):
    """The cached tokens' values, from the packed pages."""
    case = s.case
    if case["cache"] == "bf16":
        rows = s.cache.view(torch.bfloat16).reshape(-1, 576)[s.slots]
        return rows[:, :512], rows[:, 512:]
    cc, at, size = _page_layout(case)
    paper, bits = case["meta"] == "paper", 2 if case["cache"] == "c2" else 4
    pages = s.cache.reshape(-1, size)

    def region(k, width):
        return pages[:, at[k]:at[k] + PAGE * width].reshape(-1, width)[s.slots]

    def codes(raw, bits):
        """Channel 2i of a word at bits [bits i, bits (i+1)), channel 2i + 1 in the same bits of its upper half."""
        half = raw.contiguous().view(torch.int16).int().reshape(raw.shape[0], -1, 2) & 0xFFFF
        shift = torch.arange(0, 16, bits, device=DEV, dtype=torch.int32)
        return ((half[:, :, None, :] >> shift[None, None, :, None]) & ((1 << bits) - 1)).reshape(raw.shape[0], -1)

    qc, qr = codes(region(0, cc), bits), codes(region(1, 32), 4)
    if paper:
        rec = region(2, 32)
        sc, zc = rec[:, :16].contiguous().view(torch.bfloat16).float(), rec[:, 16:24].float()
        sr, zr = rec[:, 24:28].contiguous().view(torch.float32), rec[:, 28:29].float()
    else:
        mc = region(2, 32).contiguous().view(torch.float16).float().reshape(-1, 8, 2)
        mr = region(3, 4).contiguous().view(torch.float16).float()
        sc, zc, sr, zr = mc[..., 0], mc[..., 1], mr[:, :1], mr[:, 1:]
    c = (sc[..., None] * (qc.reshape(-1, 8, 64).float() - zc[..., None])).reshape(-1, 512).bfloat16()
    return c, (sr * (qr.float() - zr)).bfloat16()


def _plain(s):
    case = s.case
    if case["op"] == "attn":
        return _plain_attn(s)
    if case["op"] == "rope":
        rows = s.table[s.positions.long()]
        return {"out": _plain_rotate(s.q[..., 128:], rows[:, None, :], case["halves"])}
    out = {}
    if case["op"] == "append":
        c_new = _plain_norm(s.x, s.w)
        k_new = _plain_rotate(s.k, s.rotary[s.pos.long()], case["halves"])
        out = {"c_new": c_new, "k_new": k_new}
        paper = case["meta"] == "paper"
        if case["cache"] == "bf16":
            c, k = c_new, k_new
        else:
            c = _plain_quantized(c_new, 2 if case["cache"] == "c2" else 4, torch.bfloat16 if paper else torch.float16)
            k = _plain_quantized(k_new, 4, torch.float32 if paper else torch.float16)
        if case["prot"]:
            kept, row = _plain_protected(s)
            s.prot[row[kept]] = torch.cat([c_new, k_new], dim=1)[kept]
            out["prot"] = s.prot
            c, k = torch.where(kept[:, None], c_new, c), torch.where(kept[:, None], k_new, k)
        return dict(out, c=c, k=k)
    c, k = _plain_read(s)
    if case["prot"]:
        kept, row = _plain_protected(s)
        rows = s.prot[torch.where(kept, row, torch.zeros_like(row))]
        c, k = torch.where(kept[:, None], rows[:, :512], c), torch.where(kept[:, None], rows[:, 512:], k)
    return {"c": c, "k": k}


def run(s):
    return _run_own(s) if own else _plain(s)


# ---------------------------------------------------------------------------

def _token_bytes(case):
    if case["cache"] == "bf16":
        return 1152
    return (512 * (2 if case["cache"] == "c2" else 4) + 256) // 8 + (32 if case["meta"] == "paper" else 36)


def work(case):
    if case["op"] == "rope":
        return {"bytes": case["n"] * (case["H"] * 256 + 4 + 256), "flops": case["n"] * case["H"] * 192}
    if case["op"] == "attn":
        ql, kl = _attn_lens(case)
        pairs = 0
        for nq, nk in zip(ql, kl):
            if not case["causal"]:
                pairs += nq * nk
            else:
                seen = min(nq, nk)      # rows that see a key: nk - seen + 1 .. nk of them
                pairs += seen * (2 * nk - seen + 1) // 2
        H = case["H"]
        return {"bytes": sum(ql) * H * (384 + 256 + 4) + sum(kl) * (H * 512 + 128), "flops": 640 * pairs * H}
    new = _ragged(case, case["n"])
    T, per = sum(new), _token_bytes(case)
    kept = sum(min(n, (SINK if not case["base"] else 0) + RECENT) for n in new) if case["prot"] else 0
    if case["op"] == "gather":
        return {"bytes": (T - kept) * per + kept * 1152 + T * 1152, "flops": T * 576 * 2}
    return {"bytes": T * (1152 + 256 + 12 + 1152 + 2 * per + 1152) + kept * 2 * 1152, "flops": T * 576 * 8}


# ---------------------------------------------------------------------------
# The same in 64 bits, from the definitions.

def _exact_attn(case, seed):
    q, kv, kr = _attn_inputs(case, seed)
    ql, kl = _attn_lens(case)
    H = case["H"]
    if H * sum(a * b for a, b in zip(ql, kl)) > MOST_PAIRS:
        return None
    out = torch.zeros((sum(ql), H, 128), dtype=torch.float64, device=DEV)
    lse = torch.full((sum(ql), H), -math.inf, dtype=torch.float64, device=DEV)
    a = e = 0
    for nq, nk in zip(ql, kl):
        first = max(0, nq - nk) if case["causal"] else 0        # rows before it see nothing
        if nk and first < nq:
            seen = torch.arange(first, nq, device=DEV) + (nk - nq + 1) if case["causal"] else None
            tail = kr[e:e + nk].double()
            for h in range(H):
                x = q[a + first:a + nq, h].double()
                z = x[:, :128] @ kv[e:e + nk, h, :128].double().T.contiguous() + x[:, 128:] @ tail.T.contiguous()
                z = z / math.sqrt(192.0)
                if seen is not None:
                    z = torch.where(torch.arange(nk, device=DEV)[None] < seen[:, None], z, -math.inf)
                row = torch.logsumexp(z, dim=1)
                out[a + first:a + nq, h] = torch.exp(z - row[:, None]) @ kv[e:e + nk, h, 128:].double()
                lse[a + first:a + nq, h] = row
        a, e = a + nq, e + nk
    return {"out": out, "lse": lse}


def _exact_turn(x, angles, halves):
    """Each pair as a complex number times e^(i angle), the table's cosine and sine."""
    turn = torch.complex(angles[..., :32].double(), angles[..., 32:].double())
    x = x.double()
    pair = torch.complex(x[..., :32], x[..., 32:]) if halves else torch.view_as_complex(x.unflatten(-1, (32, 2)).contiguous())
    y = pair * turn
    return torch.cat([y.real, y.imag], dim=-1) if halves else torch.view_as_real(y).flatten(-2)


def _exact_codes(x, bits, kept_as):
    """Scale, zero-point and code of every value by the quantizer's steps, each rounded to fp32 as defined."""
    m = 2 ** bits - 1
    g = x.double().unflatten(-1, (-1, 64))
    low, high = g.min(-1, keepdim=True).values, g.max(-1, keepdim=True).values

    def fp32(v):
        return v.float().double()

    s = fp32(torch.maximum(fp32(high - low), torch.tensor(1e-8, device=DEV).double()) / m)
    z = torch.clip(torch.round(fp32(-low / s)), 0, m)
    code = torch.clip(torch.round(fp32(fp32(g / s) + z)), 0, m)
    return ((code - z) * s.to(kept_as).double()).flatten(-2)


def exact(case, seed):
    if case["op"] == "attn":
        return _exact_attn(case, seed)
    s = prepare(case, seed)
    if case["op"] == "rope":
        angles = torch.index_select(s.table, 0, s.positions)[:, None]
        return {"out": _exact_turn(s.q[..., 128:], angles, case["halves"])}
    L, at = torch.index_select(s.lens, 0, s.seq), s.pos
    held = torch.logical_or(at < SINK, at + RECENT >= L) if case["prot"] else torch.zeros_like(at, dtype=torch.bool)
    row = torch.index_select(s.prot_slot, 0, s.seq) * (SINK + RECENT) + torch.where(at < SINK, at, SINK + (at - SINK) % RECENT)
    if case["op"] == "gather":
        return _exact_gather(s, held, row)
    x = s.x.double()
    c = x * (1.0 if s.w is None else s.w.double()) / torch.sqrt(torch.sum(x ** 2, -1, keepdim=True) / 512 + _eps())
    k = _exact_turn(s.k, torch.index_select(s.rotary, 0, at), case["halves"])
    c16, k16 = c.float().bfloat16(), k.float().bfloat16()
    paper = case["meta"] == "paper"
    if case["cache"] == "bf16":
        cv, kv = c16.double(), k16.double()
    else:
        cv = _exact_codes(c16, 2 if case["cache"] == "c2" else 4, torch.bfloat16 if paper else torch.half)
        kv = _exact_codes(k16, 4, torch.float32 if paper else torch.half)
    got = {"c_new": c, "k_new": k}
    if case["prot"]:
        prot = s.prot.double()
        prot[row[held].long()] = torch.cat([c16, k16], 1).double()[held]
        got["prot"] = prot
        cv[held], kv[held] = c16.double()[held], k16.double()[held]
    return dict(got, c=cv, k=kv)


def _exact_gather(s, held, row):
    """Token by token's bytes: page, offset in it, and each channel's code by its place in the word."""
    case = s.case
    page, off = s.slots // PAGE, s.slots % PAGE
    if case["cache"] == "bf16":
        rows = s.cache.view(torch.bfloat16).double().reshape(-1, PAGE, 576)[page, off]
        return {"c": rows[:, :512], "k": rows[:, 512:]}
    cc, at, size = _page_layout(case)
    pages = s.cache.reshape(-1, size)
    bits = 2 if case["cache"] == "c2" else 4

    def value(base, width, channel, bits):
        per = 32 // bits
        word, c = channel // per, channel % per
        bit = 16 * (c % 2) + bits * (c // 2)
        byte = pages[page[:, None], base + off[:, None] * width + (word * 4 + bit // 8)[None]]
        return (byte.long() >> (bit % 8)[None]) & (2 ** bits - 1)

    def number(base, kind, size_):
        at_ = base[:, None] + torch.arange(size_, device=DEV)
        return pages[page[:, None], at_].contiguous().view(kind).double()

    ch = torch.arange(512, device=DEV)
    qc, qr = value(at[0], cc, ch, bits), value(at[1], 32, ch[:64], 4)
    if case["meta"] == "paper":
        rec = at[2] + off * 32
        sc, sr = number(rec, torch.bfloat16, 16), number(rec + 24, torch.float32, 4)
        zc, zr = number(rec + 16, torch.uint8, 8), number(rec + 28, torch.uint8, 1)
    else:
        both, one = number(at[2] + off * 32, torch.half, 32), number(at[3] + off * 4, torch.half, 4)
        sc, zc, sr, zr = both[:, 0::2], both[:, 1::2], one[:, :1], one[:, 1:]
    c = (qc - torch.repeat_interleave(zc, 64, 1)) * torch.repeat_interleave(sc, 64, 1)
    k = (qr - zr) * sr
    if case["prot"]:
        c[held], k[held] = s.prot.double()[row[held].long()].split((512, 64), 1)
    return {"c": c, "k": k}
