"""The speculative step's operators in 64 bits, for the tests.

Written from the definitions of include/mla_speculate.h; shares no code with the
library.  Cached values come from the oracle's reading of the cache's bytes.

Bounds.  A rounding is off by at most half a step: bf16 2^-8, fp16 2^-11, fp32
2^-24, relative to the value (fp16 below its normal range: 2^-25 absolute).

Attention.  A score is tau times 576 products of exact queries with keys that
carry one fp16 rounding over the low-bit cache (two in the paper's storage: its
fp32 RoPE scale is rounded to fp16 as well) and none over the BF16 cache,
summed in fp32: off by dz = tau (n_k 2^-11 + 600 2^-24) sum |q k| and a few fp32
roundings of itself.  A normalized weight is off by a factor within e^{2 dz}, by
its rounding as an operand (fp16 or bf16, numerator and sum), and by fp32 sums;
a value by one fp16 rounding; the output by its own, and a split's partial by an
fp16 one.  Weights below 2^-24 of a row's sum, and fp16 values below 2^-14, may
be lost: 2^-24 of the values' sum, and 2^-24.
"""
from __future__ import annotations

import math

import numpy as np
import torch

from oracle import paged_cache as pc

U16, U11, U24 = 2.0 ** -8, 2.0 ** -11, 2.0 ** -24
TAU = 1.0 / math.sqrt(192.0)


# --- trees

def chain(n):
    return [-1] + list(range(n - 1))


def random_tree(rng, n):
    return [-1] + [int(rng.integers(max(0, i - 4), i)) for i in range(1, n)]


def lineage_masks(parents):
    """Bit j of mask i: j is i or above it."""
    masks = []
    for i, p in enumerate(parents):
        masks.append((1 << i) | (masks[p] if p >= 0 else 0))
    return masks


def mask_tensor(masks, device="cpu"):
    return torch.tensor([m - (1 << 64) if m >> 63 else m for m in masks], dtype=torch.int64, device=device)


# --- caches

KINDS = ("c4", "c2", "c4p", "c2p", "bf16")


def oracle_format(kind, page_size=64):
    return pc.CacheFormat(c_bits=2 if kind.startswith("c2") else 4, page_size=page_size, meta="paper" if kind.endswith("p") else "fp16")


def library_format(kind, page_size=64):
    from paper_2609_36760_amd import _binding as mb
    return mb.cache_format(c_bits=2 if kind.startswith("c2") else 4, page_size=page_size,
                           meta=mb.MLA_META_PAPER if kind.endswith("p") else mb.MLA_META_FP16)


def page_bytes(kind, page_size=64):
    return page_size * 1152 if kind == "bf16" else oracle_format(kind, page_size).page_bytes


def block_table(rng, lens, page_size, spare=2):
    """Pages of sequences of these lengths in random order, some pages unused; int32 [B, most], and their number."""
    counts = [-(-n // page_size) for n in lens]
    ids = rng.permutation(sum(counts) + spare).astype(np.int32)
    table = np.zeros((len(lens), max(counts + [1]) + 1), np.int32)
    at = 0
    for b, k in enumerate(counts):
        table[b, :k] = ids[at:at + k]
        at += k
    return table, sum(counts) + spare


def cached_values(cache, kind, table_row, n, page_size=64):
    """The first n tokens as float64 [n, 576] from the cache's bytes (uint8 array)."""
    pages = cache.reshape(-1, page_bytes(kind, page_size))[table_row[:-(-n // page_size)].astype(np.int64)]
    if kind == "bf16":
        rows = np.ascontiguousarray(pages).view(np.uint16).reshape(-1, 576)[:n]
        return (rows.astype(np.uint32) << np.uint32(16)).view(np.float32).astype(np.float64)
    fmt = oracle_format(kind, page_size)
    c, k = pc.decode_blocks(fmt, pc.page_blocks(fmt, pages, n))
    return np.concatenate([c, k], axis=1).astype(np.float64)


# --- attention

class TreeRows:
    """Outputs, lse and their bounds of one sequence's rows (float64 [n, H, ..]).

    ``x``: cached values [ctx + n, 576]; keys in ``bad`` (indexes) have a channel that is not finite."""

    def __init__(self, q, x, ctx, masks, kind, split=True, tau=TAU, bad=()):
        n, H = q.shape[:2]
        T = x.shape[0]
        low = kind != "bf16"
        rounded = (2.0 if kind.endswith("p") else 1.0) * U11 if low else 0.0
        weights = U11 if low else U16
        x = np.array(x)
        x[list(bad)] = 0.0
        self.out = np.zeros((n, H, 512))
        self.lse = np.full((n, H), -np.inf)
        self.out_bound = np.full((n, H, 512), 1e-30)
        self.lse_bound = np.zeros((n, H))
        for i in range(n):
            seen = np.ones(T, bool)
            for j in range(n):
                seen[ctx + j] = (masks[i] >> j) & 1
            if not seen.any():
                continue
            if any(seen[t] for t in bad):
                self.out[i], self.lse[i] = np.nan, np.nan
                continue
            k = x[seen]
            z = tau * (q[i] @ k.T)
            dz = (tau * (rounded + 600 * U24) * (np.abs(q[i]) @ np.abs(k).T) + 4 * U24 * np.abs(z)).max(1, keepdims=True)
            top = z.max(1, keepdims=True)
            lse = top + np.log(np.exp(z - top).sum(1, keepdims=True))
            w = np.exp(z - lse)
            v = k[:, :512]
            self.out[i], self.lse[i] = w @ v, lse[:, 0]
            spread = w @ np.abs(v)
            delta = np.expm1(2.0 * dz) + 2.0 * weights + (U11 if low else 0.0) + (U11 if split else 0.0) + 2.0 ** -20 + T * U24
            lost = (np.abs(v).sum(0)[None] * U24 + U24) if low or split else 0.0
            self.out_bound[i] = 1.02 * (U16 * np.abs(self.out[i]) + delta * spread) + lost + 1e-30
            self.lse_bound[i] = (dz + weights + 2.0 ** -20 + T * U24 + 4 * U24 * np.abs(lse))[:, 0]

    def check(self, out, lse, what):
        """``out`` float [n, H, 512], ``lse`` [n, H] or None (numpy)."""
        out = out.astype(np.float64)
        fine = np.isfinite(self.out)
        assert np.array_equal(np.isnan(self.out), np.isnan(out)), f"{what}: NaN in other places"
        ratio = (np.abs(out - self.out) / self.out_bound)[fine]
        worst = float(ratio.max()) if ratio.size else 0.0
        assert worst <= 1.0, f"{what}: output off by {worst:.3g} of the bound"
        if lse is not None:
            lse = lse.astype(np.float64)
            empty = self.lse == -np.inf
            assert np.array_equal(empty, lse == -np.inf), f"{what}: rows without keys"
            assert np.array_equal(np.isnan(self.lse), np.isnan(lse)), f"{what}: lse NaN"
            fine = np.isfinite(self.lse)
            r = (np.abs(lse - np.where(fine, self.lse, 0.0)) / np.maximum(self.lse_bound, 1e-30))[fine]
            assert r.size == 0 or r.max() <= 1.0, f"{what}: lse off by {float(r.max()):.3g} of the bound"
        return worst


# --- verification

def softmax64(logits, t):
    """p of one row, or None for a row that cannot be used; t = 0: all on the first largest."""
    l = np.asarray(logits, np.float64)
    if np.isnan(l).any() or (l == np.inf).any() or not (l > -np.inf).any():
        return None
    if t == 0.0:
        p = np.zeros_like(l)
        p[int(np.argmax(l))] = 1.0
        return p
    with np.errstate(over="ignore"):
        w = np.exp((l - l.max()) / t)
    return w / math.fsum(w)


def verify(logits, tokens, parents, u_accept, u_draw, t, probs=None):
    """(path, emitted, logprobs) of one sequence: float rows [n, V], a list each."""
    n, V = len(parents), logits.shape[1]
    path, emitted, logprobs = [], [], []
    if n == 0:
        return path, emitted, logprobs
    v = 0
    while True:
        path.append(v)
        p = softmax64(logits[v], t)
        if p is None:
            return path, emitted + [-1], logprobs + [0.0]
        r = p.copy()
        taken = None
        for i in range(v + 1, n):
            if parents[i] != v:
                continue
            x, u = int(tokens[i]), float(u_accept[i])
            real = 0 <= x < V
            if t == 0.0:
                yes = real and r[x] > 0
            elif probs is None:
                yes = real and u * math.fsum(r) < r[x]
                if not yes and real:
                    r[x] = 0.0
            else:
                q = np.asarray(probs[v], np.float64)
                yes = real and u * q[x] < r[x]
                if not yes:
                    with np.errstate(invalid="ignore"):
                        left = np.where(r - q > 0, r - q, 0.0)
                    if math.fsum(left) > 0:
                        r = left / math.fsum(left)
            if yes:
                taken = i
                break
        if taken is None:
            up = np.cumsum(r)
            x = int(np.argmax((up > float(u_draw) * up[-1]) & (r > 0)))
            if not ((up > float(u_draw) * up[-1]) & (r > 0)).any():
                x = int(np.nonzero(r)[0][-1])
        else:
            x = int(tokens[taken])
        emitted.append(x)
        logprobs.append(0.0 if t == 0.0 else math.log(p[x]))
        if taken is None:
            return path, emitted, logprobs
        v = taken


# --- commit

def commit(caches, kind, page_size, table, num_pages, ctx, path, keep, max_nodes):
    """The caches (uint8 [layers, bytes]) after the commit, and the new lengths."""
    caches = caches.copy()
    if kind == "bf16":
        sizes, offs, size = [1152], [0], page_size * 1152
    else:
        fmt = oracle_format(kind, page_size)
        sizes, offs, size = fmt.region_sizes(), fmt.region_offsets(), fmt.page_bytes
    for cache in caches:
        pages = cache[:num_pages * size].reshape(num_pages, size)
        for b in range(len(ctx)):
            rows = []
            for k in range(min(max(int(keep[b]), 0), max_nodes)):
                node = int(path[b][k])
                ends = []
                for pos in (int(ctx[b]) + node, int(ctx[b]) + k):
                    page, off = divmod(pos, page_size)
                    ok = 0 <= node < max_nodes and page < table.shape[1] and 0 <= table[b, page] < num_pages
                    ends.append((table[b, page], off) if ok else None)
                if None not in ends:
                    (p, o), to = ends
                    rows.append((to, [pages[p, a + o * s:a + (o + 1) * s].copy() for a, s in zip(offs, sizes)]))
            for (p, o), parts in rows:
                for a, s, part in zip(offs, sizes, parts):
                    pages[p, a + o * s:a + (o + 1) * s] = part
    return caches, np.asarray(ctx) + np.clip(keep, 0, max_nodes)
