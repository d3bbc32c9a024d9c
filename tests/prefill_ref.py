"""The prompt-side operators in 64 bits, for the tests (torch, on the CPU or GPU).

Written from the definitions of include/mla_prefill.h; shares no code with the
library.
"""
from __future__ import annotations

import math

import numpy as np
import torch

U16 = 2.0 ** -8         # half a bf16 step, relative to the value
U32 = 2.0 ** -24


def rotation_table(n, scale=1.0):
    theta = 10000.0 ** (-np.arange(32) / 32.0) * scale
    a = np.arange(n)[:, None] * theta
    return torch.from_numpy(np.concatenate([np.cos(a), np.sin(a)], axis=1).astype(np.float32))


def rotate(x, rows, halves):
    """bf16 ``x`` [..., 64] rotated by fp32 table rows [..., 64], as bf16."""
    cos, sin = rows[..., :32].double(), rows[..., 32:].double()
    x = x.double()
    if halves:
        a, b = x[..., :32], x[..., 32:]
        y = torch.cat([a * cos - b * sin, a * sin + b * cos], dim=-1)
    else:
        a, b = x[..., ::2], x[..., 1::2]
        y = torch.stack([a * cos - b * sin, a * sin + b * cos], dim=-1).flatten(-2)
    return y.float().bfloat16()


def rms_norm(x, weight, eps):
    """bf16 ``x`` [n, 512] normalized, as bf16; ``eps`` as the fp32 value a caller passes."""
    d = x.double()
    w = 1.0 if weight is None else weight.double()
    r = 1.0 / torch.sqrt((d * d).sum(-1, keepdim=True) / 512.0 + float(np.float32(eps)))
    return (d * w * r).float().bfloat16()


def bits(t):
    """bf16 tensor as uint16 bit patterns (numpy)."""
    return t.cpu().contiguous().view(torch.int16).numpy().view(np.uint16)


class Attended:
    """Outputs, lse and their bounds of one sequence's rows (float64, [q, H, ...])."""

    def __init__(self, q_nope, q_rope, k_nope, k_rope, v, causal, tau):
        nq, H = q_nope.shape[:2]
        nk = k_nope.shape[0]
        dev = q_nope.device
        self.out = torch.zeros((nq, H, 128), dtype=torch.float64, device=dev)
        self.lse = torch.full((nq, H), -math.inf, dtype=torch.float64, device=dev)
        self.out_bound = torch.zeros_like(self.out)
        self.lse_bound = torch.zeros_like(self.lse)
        seen = torch.full((nq,), nk, device=dev)
        if causal:
            seen = (torch.arange(nq, device=dev) + nk - nq + 1).clamp(min=0)
        hidden = torch.arange(nk, device=dev)[None, :] >= seen[:, None]
        for h in range(H):
            if nk == 0:
                continue
            q = torch.cat([q_nope[:, h], q_rope[:, h]], dim=-1).double()
            k = torch.cat([k_nope[:, h], k_rope], dim=-1).double()
            val = v[:, h].double()
            z = tau * (q @ k.T.contiguous())
            # fp32 scores: 192 products and sums, the scale and the difference from the reference
            mass = q.abs() @ k.abs().T.contiguous()
            dz = U32 * (tau * 256.0 * mass + 4.0 * z.abs())
            z = z.masked_fill(hidden, -math.inf)
            dz = dz.masked_fill(hidden, 0.0).nan_to_num(0.0).amax(1, keepdim=True)
            some = (seen > 0)[:, None]
            lse = torch.logsumexp(z, dim=1, keepdim=True)
            w = torch.exp(z - lse).masked_fill(hidden, 0.0)
            # hidden keys have no part, whatever they hold
            o = torch.where(hidden[:, :, None], 0.0, w[:, :, None] * val[None]).sum(1) if not torch.isfinite(val).all() \
                else w @ val
            self.out[:, h] = torch.where(some, o, 0.0)
            self.lse[:, h] = torch.where(some, lse, -math.inf)[:, 0]
            # weights: bf16 rounding of each (twice, should their sum be taken of the rounded ones), the scores' error
            # (numerator and sum), exp2 and fp32 sums (some 2^-20); then the output's own rounding
            spread = w @ val.nan_to_num(0.0, 0.0, 0.0).abs()
            delta = 2.0 * U16 + 4.0 * dz + 2.0 ** -20 + nk * U32
            self.out_bound[:, h] = 1.01 * (U16 * self.out[:, h].nan_to_num(0.0, 0.0, 0.0).abs() + delta * spread) + 1e-30
            self.lse_bound[:, h] = (2.0 * dz + 2.0 ** -20 + nk * U32 + 4.0 * U32 * lse.nan_to_num(0.0, 0.0, 0.0).abs())[:, 0]

    def check(self, out, lse, what):
        got = out.double()
        fine = torch.isfinite(self.out)
        assert torch.equal(torch.isnan(self.out), torch.isnan(got)), f"{what}: NaN in other places"
        assert torch.equal(self.out[~fine & ~self.out.isnan()], got[~fine & ~got.isnan()]), f"{what}: infinities"
        ratio = ((got - self.out).abs() / self.out_bound.clamp(min=1e-30))[fine]
        if ratio.numel():
            assert ratio.max() <= 1.0, f"{what}: output off by {float(ratio.max()):.3g} of the bound"
        if lse is not None:
            l = lse.double()
            empty = self.lse == -math.inf
            assert torch.equal(empty, l == -math.inf), f"{what}: rows without keys"
            fine = torch.isfinite(self.lse)
            assert torch.equal(torch.isnan(self.lse), torch.isnan(l)), f"{what}: lse NaN"
            r = ((l - self.lse).abs() / self.lse_bound)[fine]
            if r.numel():
                assert r.max() <= 1.0, f"{what}: lse off by {float(r.max()):.3g} of the bound"
        return float(ratio.max()) if ratio.numel() else 0.0
