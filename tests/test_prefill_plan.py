"""The planner of the expanded attention and the refusals of mla_prefill.h
(CPU only; no GPU work is launched).

A plan's work items must cover every (row, visible key) pair exactly once,
longest first, with every split's partial merged once; lengths, starts and
every argument that a call cannot take are refused before any HIP call.
"""
import ctypes
import os
import re

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def mp():
    from paper_2609_36760_amd import _binding, _prefill
    if not os.path.exists(_binding.LIB_PATH):
        pytest.skip("libmla_lowbit.so not built (run __graft_entry__.build())")
    _prefill.library()
    return _prefill


def test_exports_every_declared_symbol(mp):
    text = open(os.path.join(ROOT, "include", "mla_prefill.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    assert sorted(set(re.findall(r"\bint (mla_[a-z0-9_]+)\s*\(", text))) == sorted(mp.SYMBOLS)


def test_public_names(mp):
    import paper_2609_36760_amd as pkg
    for name in mp.SYMBOLS:
        assert getattr(pkg, name) is getattr(mp, name)


PLANS = [
    # (q_lens, kv_lens, H, causal)
    ([1], [1], 1, True), ([64], [64], 16, True), ([1000, 3, 129], [1000, 70, 5000], 4, True),
    ([5, 0, 3], [2, 0, 0], 2, True), ([200], [100], 3, True), ([7], [30000], 2, True), ([300], [20000], 1, False),
    ([1] * 40, list(range(0, 4000, 100)), 8, True), ([257, 31], [0, 900], 16, False), ([], [], 1, True),
    ([1, 1], [100000, 3], 16, True), ([1500, 700, 3000, 20], [1500, 700, 3000, 20], 64, True),
    ([256] * 70, [300] * 70, 3, False), ([2000, 0, 900], [0, 400, 50], 24, True),
]


def check_order(items, work, rest, info, H):
    """Items the longest first; blocks of 256 rows sequence by sequence, and dealt out to lists."""
    if info.rows != 256:
        assert work == sorted(work, reverse=True) and len(rest) == 0
        return
    seqs = items[:, 7].tolist()
    runs = [i for i in range(len(seqs)) if i == 0 or seqs[i] != seqs[i - 1]]
    assert len(runs) == len(set(seqs))
    for a, b in zip(runs, runs[1:] + [len(seqs)]):
        assert work[a:b] == sorted(work[a:b], reverse=True)
    heads, most = (H // 8, 32) if H % 8 == 0 else (H, 256)
    lists = min(most, heads * len(items))
    first, entries = rest[:lists + 1], rest[lists + 1:]
    entries = np.where(entries < 0, ~entries, entries)          # (complement: from the last tile down)
    assert first[0] == 0 and first[-1] == len(entries) and (np.diff(first) > 0).all()
    assert sorted(entries.tolist()) == list(range(heads * len(items)))
    # taken as they come: no list waits longer than its last entry
    load = [sum(5 + work[e // heads] for e in entries[a:b]) for a, b in zip(first, first[1:])]
    last = [5 + work[entries[b - 1] // heads] for b in first[1:]]
    assert all(n - t <= min(load) for n, t in zip(load, last))


@pytest.mark.parametrize("q,kv,H,causal", PLANS)
def test_plan_covers_every_pair_once(mp, q, kv, H, causal):
    plan, info = mp.mla_plan_prefill(q, kv, H, causal)
    records = 8 * (info.num_items + info.num_merges)
    rec = plan[:records].reshape(-1, 8)
    items, merges = rec[:info.num_items], rec[info.num_items:]
    assert info.total_q == sum(q) and info.total_kv == sum(kv) and len(merges) == info.num_merges
    q0, k0 = np.cumsum([0] + list(q)), np.cumsum([0] + list(kv))
    seq_of = np.repeat(np.arange(len(q)), q)
    seen = np.zeros(sum(q), np.int64)                   # keys covered of each row
    reach = [[] for _ in range(sum(q))]
    work = []
    for q_row, rows, kv_row, key0, key1, seen0, part, _ in items.tolist():
        assert 1 <= rows <= info.rows and 0 <= key0 <= key1
        work.append((key1 - key0 + 63) // 64)
        for r in range(rows):
            b = seq_of[q_row + r]
            assert b == seq_of[q_row] and kv_row == k0[b]
            i = q_row + r - q0[b]
            limit = kv[b] if not causal else max(0, min(kv[b], kv[b] - q[b] + i + 1))
            lo, hi = key0, max(key0, min(key1, seen0 + r))
            assert hi <= max(limit, key0)
            reach[q_row + r].append((lo, hi, limit))
    check_order(items, work, plan[records:], info, H)
    for spans in reach:
        spans.sort()
        assert spans
        at = 0
        for lo, hi, limit in spans:
            if hi > lo:
                assert lo == at
                at = hi
        assert at == spans[0][2]
    # every partial belongs to one merge, whose block is the item's
    owner = {}
    for q_row, rows, part0, n, _, kv_len, _, _ in merges.tolist():
        assert n > 1
        for p in range(part0, part0 + n):
            assert p not in owner
            owner[p] = (q_row, rows, kv_len)
    parts = {int(x[6]): (int(x[0]), int(x[1])) for x in items if x[6] >= 0}
    assert sorted(parts) == sorted(owner) == list(range(info.num_parts))
    for p, block in parts.items():
        assert owner[p][:2] == block and owner[p][2] == kv[seq_of[block[0]]]
    whole = [int(x[0]) for x in items if x[6] < 0]
    assert len(set(whole)) == len(whole) and not set(whole) & {int(x[0]) for x in merges}
    assert info.part_rows == max((m[1] for m in merges.tolist()), default=0)
    assert info.workspace_bytes == info.num_parts * H * info.part_rows * (128 * 4 + 8)


def test_plan_starts(mp):
    plan, info = mp.mla_plan_prefill([3, 2], [5, 9], 2, True, q_starts=[10, 0], kv_starts=[0, 16])
    assert (info.total_q, info.total_kv) == (13, 25)
    rows = sorted((r[0], r[1], r[2]) for r in plan.reshape(-1, 8).tolist())
    assert rows == [(0, 2, 16), (10, 3, 0)]
    mp.mla_plan_prefill([3, 2], [5, 5], 2, True, q_starts=[0, 3], kv_starts=[0, 0])     # keys may be shared
    mp.mla_plan_prefill([3, 0], [5, 5], 2, True, q_starts=[0, 1])


@pytest.mark.parametrize("q,kv,H,more,status", [
    ([-1], [3], 2, {}, 1), ([3], [-1], 2, {}, 1), ([3], [3], 0, {}, 1), ([3], [3], -2, {}, 1),
    ([3, 3], [3, 3], 1, dict(q_starts=[0, 2]), 1), ([3], [3], 1, dict(q_starts=[-1]), 1),
    ([3], [3], 1, dict(kv_starts=[-1]), 1), ([(1 << 30) + 1], [3], 1, {}, 2), ([3], [(1 << 30) + 1], 1, {}, 2),
    ([1 << 30], [1], 128, {}, 2), ([1], [1], 1 << 30, {}, 2),
])
def test_plan_refusals(mp, q, kv, H, more, status):
    from paper_2609_36760_amd import _binding as mb
    with pytest.raises(mb.MlaError) as e:
        mp.mla_plan_prefill(q, kv, H, True, **more)
    assert e.value.status == status


def test_plan_capacity_and_nulls(mp):
    lib = mp.library()
    info = mp.mla_prefill_plan()
    q = np.array([200], np.int32)
    buf = np.zeros(64, np.int32)
    p, i = q.ctypes.data, ctypes.byref(info)
    assert lib.mla_plan_prefill(p, p, None, None, 1, 2, 1, None, 0, i) == 0
    n = info.plan_ints
    assert 8 <= n < 64
    assert lib.mla_plan_prefill(p, p, None, None, 1, 2, 1, buf.ctypes.data, n - 1, i) == 1
    assert info.plan_ints == n and not buf.any()
    assert lib.mla_plan_prefill(p, p, None, None, 1, 2, 1, buf.ctypes.data, n, i) == 0
    assert buf[:n].any() and not buf[n:].any()
    assert lib.mla_plan_prefill(p, p, None, None, 1, 2, 1, None, 0, None) == 1
    assert lib.mla_plan_prefill(None, p, None, None, 1, 2, 1, None, 0, i) == 1
    assert lib.mla_plan_prefill(p, p, None, None, -1, 2, 1, None, 0, i) == 1
    assert lib.mla_plan_prefill(p, p, None, None, 1, 2, 2, None, 0, i) == 1


def _attn(mp, q=(40,), kv=(5000,), H=2, info_over=None, **over):
    _, info = mp.mla_plan_prefill(list(q), list(kv), H, True)
    for k, v in (info_over or {}).items():
        setattr(info, k, v)
    rows = {n: mp.mla_head_rows(4096, 384, 192) for n in ("q_nope", "q_rope", "k_nope", "k_rope", "v")}
    a = dict(plan=256, scale=0.07, out=256, out_t=H * 128, out_h=128, lse=None, workspace=256, size=info.workspace_bytes)
    for k, v in over.items():
        if k in rows:
            rows[k] = None if v is None else mp.mla_head_rows(*v)
        else:
            a[k] = v
    ptrs = [None if rows[n] is None else ctypes.byref(rows[n]) for n in ("q_nope", "q_rope", "k_nope", "k_rope", "v")]
    return mp.library().mla_prefill_attn(ctypes.byref(info), a["plan"], *ptrs, a["scale"], a["out"], a["out_t"], a["out_h"],
                                         a["lse"], a["workspace"], a["size"], None)


@pytest.mark.parametrize("over,status", [
    (dict(plan=None), 1), (dict(plan=8), 2), (dict(out=None), 1), (dict(out=8), 2), (dict(scale=0.0), 1),
    (dict(scale=float("nan")), 1), (dict(scale=float("inf")), 1), (dict(scale=-1.0), 1),
    (dict(q_nope=None), 1), (dict(q_nope=(None, 384, 192)), 1), (dict(q_rope=(4096, -8, 192)), 1),
    (dict(k_nope=(4096, 384, -8)), 1), (dict(k_nope=(4096, 380, 192)), 2), (dict(k_nope=(4096, 384, 196)), 2),
    (dict(v=(4104, 384, 192)), 2), (dict(v=(4096, 1 << 24, 192)), 2), (dict(v=(4096, 384, 1 << 24)), 2),
    (dict(k_rope=(None, 64, 0)), 1), (dict(k_rope=(4096, 60, 0)), 2),
    (dict(out_t=128, out_h=128), 1), (dict(out_t=256, out_h=64), 1), (dict(out_t=-256), 1), (dict(out_t=260), 2),
    (dict(workspace=None), 1), (dict(size=0), 1), (dict(workspace=264), 2),
    (dict(info_over=dict(rows=64)), 1), (dict(info_over=dict(part_rows=0)), 1), (dict(info_over=dict(part_rows=129)), 1), (dict(info_over=dict(rows=0)), 1), (dict(info_over=dict(H=0)), 1),
    (dict(info_over=dict(plan_ints=8)), 1), (dict(info_over=dict(num_items=-1)), 1), (dict(info_over=dict(total_q=0)), 1),
    (dict(info_over=dict(workspace_bytes=0)), 1), (dict(info_over=dict(total_kv=1 << 31)), 1),
])
def test_attention_refusals(mp, over, status):
    assert _attn(mp, **over) == status


def test_attention_without_rows_is_a_no_op(mp):
    assert _attn(mp, q=(), kv=(), plan=None, out=None) == 0
    assert _attn(mp, q=(0, 0), kv=(7, 0), plan=None, out=None, q_nope=None) == 0


def _fmt(mb, name=None):
    return {None: mb.cache_format(), "c3": mb.cache_format(c_bits=3), "p48": mb.cache_format(page_size=48)}[name]


@pytest.mark.parametrize("over,status", [
    (dict(rot=None), 1), (dict(table=None), 1), (dict(table=8), 2), (dict(positions_n=0), 1), (dict(layout=2), 1),
    (dict(eps=0.0), 1), (dict(eps=float("nan")), 1), (dict(eps=-1e-6), 1), (dict(weight=8), 2),
    (dict(c=None), 1), (dict(k=None), 1), (dict(pos=None), 1), (dict(slots=None), 1), (dict(cache=None), 1),
    (dict(c=18), 2), (dict(cs=500), 1), (dict(cs=516), 2), (dict(ks=60), 1), (dict(ks=68), 2), (dict(n=-1), 1),
    (dict(cache=272), 1), (dict(pages=0), 1), (dict(n=(1 << 25) + 1), 2), (dict(c_out=8), 2),
    (dict(c_out=4096, cos=500), 1), (dict(c_out=4096, cos=516), 2), (dict(k_out=8), 2), (dict(k_out=4096, kos=56), 1),
    (dict(c_out=16, cos=520), 1), (dict(k_out=32, kos=72), 1), (dict(fmt="c3"), 1), (dict(fmt="p48"), 2),
    (dict(n=0, c=None, cache=None), 0),
])
@pytest.mark.parametrize("kind", ["lowbit", "bf16", "protected"])
def test_append_refusals(mp, over, status, kind):
    from paper_2609_36760_amd import _binding as mb
    if kind == "bf16" and over.get("fmt") == "c3":
        pytest.skip("the BF16 cache has no codes")
    a = dict(rot=1, table=16, positions_n=10, layout=0, eps=1e-6, weight=None, c=16, cs=512, k=32, ks=64, pos=16, slots=16,
             n=4, cache=256, pages=2, c_out=None, cos=512, k_out=None, kos=64, fmt=None)
    a.update(over)
    fmt = _fmt(mb, a["fmt"])
    rot = mp.mla_rotation(a["table"], a["positions_n"], a["layout"])
    norm = mp.mla_rms_norm(a["weight"], a["eps"])
    args = [ctypes.byref(norm), None if a["rot"] is None else ctypes.byref(rot), a["c"], a["cs"], a["k"], a["ks"],
            a["pos"], a["slots"], a["n"], a["cache"], a["pages"]]
    out = [a["c_out"], a["cos"], a["k_out"], a["kos"], None]
    lib = mp.library()
    if kind == "protected":
        pol = mb.protect_policy()
        got = lib.mla_lowbit_norm_rope_append_protected(ctypes.byref(fmt), ctypes.byref(pol), *args, 16, 16, 16, 1, 16, 1, *out)
    else:
        got = getattr(lib, f"mla_{kind}_norm_rope_append")(ctypes.byref(fmt), *args, *out)
    assert got == status


@pytest.mark.parametrize("over,status", [
    (dict(policy=None), 1), (dict(sink=0, recent=0), 1), (dict(seq=None), 1), (dict(lens=None), 1), (dict(slot=None), 1),
    (dict(prot=None), 1), (dict(prot=8), 2), (dict(B=0), 1), (dict(B=-1), 1), (dict(num_prot=0), 1), (dict(num_prot=-1), 1),
])
def test_protection_refusals(mp, over, status):
    from paper_2609_36760_amd import _binding as mb
    a = dict(policy=1, sink=4, recent=128, seq=16, lens=16, slot=16, B=1, prot=16, num_prot=1)
    a.update(over)
    fmt, rot, pol = mb.cache_format(), mp.mla_rotation(16, 10, 0), mb.protect_policy(a["sink"], a["recent"])
    p = None if a["policy"] is None else ctypes.byref(pol)
    lib = mp.library()
    assert lib.mla_lowbit_norm_rope_append_protected(
        ctypes.byref(fmt), p, None, ctypes.byref(rot), 16, 512, 16, 64, 16, 16, 4, 256, 2, a["seq"], a["lens"], a["slot"],
        a["B"], a["prot"], a["num_prot"], None, 0, None, 0, None) == status
    if "seq" not in over and over.get("B") != 0:       # (no sequences: nothing to read)
        assert lib.mla_lowbit_gather_protected(
            ctypes.byref(fmt), p, 256, 2, 16, 1, None, 16, a["B"], 4, a["lens"], a["prot"], a["num_prot"], a["slot"], 16, 512,
            16, 64, None) == status


@pytest.mark.parametrize("over,status", [
    (dict(cache=None), 1), (dict(cache=272), 1), (dict(pages=0), 1), (dict(pages=-1), 1), (dict(table=None), 1),
    (dict(width=0), 1), (dict(cu=None), 1), (dict(B=-1), 1), (dict(n=-1), 1), (dict(n=(1 << 25) + 1), 2),
    (dict(c=None), 1), (dict(k=None), 1), (dict(c=8), 2), (dict(cs=508), 1), (dict(cs=516), 2), (dict(ks=32), 1),
    (dict(k=40), 2), (dict(fmt="c3"), 1), (dict(fmt="p48"), 2), (dict(n=0, c=None, cache=None), 0), (dict(B=0, cu=None), 0),
])
@pytest.mark.parametrize("kind", ["lowbit", "bf16"])
def test_gather_refusals(mp, over, status, kind):
    from paper_2609_36760_amd import _binding as mb
    if kind == "bf16" and over.get("fmt") == "c3":
        pytest.skip("the BF16 cache has no codes")
    a = dict(cache=256, pages=2, table=16, width=3, cu=16, B=1, n=4, c=16, cs=512, k=16, ks=64, fmt=None)
    a.update(over)
    fmt = _fmt(mb, a["fmt"])
    got = getattr(mp.library(), f"mla_{kind}_gather")(ctypes.byref(fmt), a["cache"], a["pages"], a["table"], a["width"], None,
                                                      a["cu"], a["B"], a["n"], a["c"], a["cs"], a["k"], a["ks"], None)
    assert got == status


@pytest.mark.parametrize("over,status", [
    (dict(rot=None), 1), (dict(q=None), 1), (dict(pos=None), 1), (dict(out=None), 1), (dict(n=-1), 1), (dict(H=0), 1),
    (dict(q=8), 2), (dict(out=8), 2), (dict(qt=-8), 1), (dict(qh=196), 2), (dict(oh=-64), 1), (dict(ot=4), 2),
    (dict(ot=64, oh=64), 1), (dict(out=16, q=16), 1), (dict(n=1 << 30, H=4, ot=256, oh=64), 2), (dict(n=0, q=None), 0),
])
def test_rope_refusals(mp, over, status):
    a = dict(rot=1, q=16, qt=384, qh=192, pos=16, n=4, H=2, out=4096, ot=128, oh=64)
    a.update(over)
    rot = mp.mla_rotation(16, 10, 0)
    assert mp.library().mla_rope_queries(None if a["rot"] is None else ctypes.byref(rot), a["q"], a["qt"], a["qh"], a["pos"],
                                         a["n"], a["H"], a["out"], a["ot"], a["oh"], None) == status
