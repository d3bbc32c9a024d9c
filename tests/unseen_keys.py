"""Support of the expanded attention's tests on extreme inputs: the 64-bit
formula with bounds that stay finite, and the splits of a plan that some rows
of a wave see nothing of.

Unlike ``prefill_ref.Attended``, whose bounds a visible infinite score makes
infinite, the bounds here are taken over the keys that a row sees with a finite
score (a key that scores -inf weighs nothing), and are asserted to be finite.
"""
from __future__ import annotations

import math

import torch

from prefill_ref import U16, U32

LOST = 2.0 ** -66       # what a key may lose by its weight, or its product with a value, leaving fp32's range


def split_edges(plan, info):
    """(first query row, block rows, key0, rows that see nothing) of every split whose last-named rows share a wave
    with rows that see something of it."""
    wave_rows = 32 if info.rows == 128 else 64
    found = []
    for q_row, rows, _, key0, key1, seen0, part, _ in plan[:8 * info.num_items].reshape(-1, 8).tolist():
        blind = [r for r in range(rows) if min(key1, seen0 + r) <= key0]
        if part >= 0 and blind and len(blind) < rows and len(blind) % wave_rows:
            found.append((q_row, rows, key0, blind))
    return found


def check_finite_case(c, heads, what):
    """Every output and lse of the call ``c`` (``test_gpu_prefill.Call``), whose visible scores are finite or -inf and
    whose values are finite, against the formula."""
    torch.cuda.synchronize()
    worst = 0.0
    for b, (nq, nk) in enumerate(zip(c.q_lens, c.kv_lens)):
        a, e = c.q0[b], c.k0[b]
        if nq == 0:
            continue
        seen = torch.full((nq,), nk, device="cuda")
        if c.causal:
            seen = (torch.arange(nq, device="cuda") + nk - nq + 1).clamp(min=0)
        hidden = torch.arange(nk, device="cuda")[None] >= seen[:, None]
        for h in heads:
            q = torch.cat([c.q_nope[a:a + nq, h], c.q_rope[a:a + nq, h]], -1).double()
            k = torch.cat([c.k_nope[e:e + nk, h], c.k_rope[e:e + nk]], -1).double()
            v = c.v[e:e + nk, h].double()
            tau = 1.0 / math.sqrt(192.0)
            z = (tau * (q @ k.T.contiguous())).masked_fill(hidden, -math.inf)
            counts = z > -math.inf
            assert torch.isfinite(z[counts]).all() and torch.isfinite(v).all() and not z.isnan().any()
            some = counts.any(1, keepdim=True)
            lse = torch.where(some, torch.logsumexp(z.masked_fill(~some, 0.0), 1, keepdim=True), -math.inf)
            w = torch.where(counts, torch.exp(z - lse.masked_fill(~some, 0.0)), 0.0)
            out = w @ v
            # fp32 scores: 192 products and sums, the scale and the difference from the reference (which lies within
            # 2^+-60 of the row's sum: 42 natural units), of the keys that count
            dz = U32 * (256.0 * tau * (q.abs() @ k.abs().T.contiguous()) + 4.0 * (z.abs() + 42.0))
            dz = torch.where(counts, dz, 0.0).amax(1, keepdim=True)
            # as in prefill_ref.Attended: weights in bf16 (twice, should their sum be taken of the rounded ones), scores,
            # exp2 and fp32 sums; the output's rounding; what leaves fp32's range
            delta = 2.0 * U16 + 4.0 * dz + 2.0 ** -20 + nk * U32
            out_bound = 1.01 * (U16 * out.abs() + delta * (w @ v.abs())) + LOST * (nk + v.abs().sum(0, keepdim=True))
            lse_bound = 2.0 * dz + 2.0 ** -20 + nk * (U32 + LOST) + 4.0 * U32 * (lse.masked_fill(~some, 0.0).abs() + 42.0)
            assert torch.isfinite(out_bound).all() and torch.isfinite(lse_bound).all()
            got, got_lse = c.out[a:a + nq, h].double(), c.lse[a:a + nq, h].double()
            assert torch.isfinite(got).all(), f"{what}, head {h}: {int((~torch.isfinite(got)).any(1).sum())} rows are not finite"
            r = float(((got - out).abs() / out_bound).max())
            assert r <= 1.0, f"{what}, head {h}: output off by {r:.3g} of the bound"
            none = ~some[:, 0]
            assert torch.equal(none, got_lse == -math.inf) and bool((got[none] == 0.0).all()), f"{what}: rows without keys"
            r = max([r] + ((got_lse - lse[:, 0]).abs() / lse_bound[:, 0])[~none].tolist())
            assert r <= 1.0, f"{what}, head {h}: off by {r:.3g} of the bound"
            worst = max(worst, r)
    print(f"  {what}: worst {worst:.2f} of its bound", flush=True)
