"""Verification after rejections that leave little of a row (GPU): outcomes are those of 64
bits where a random number is further than 1e-12 / s from a border, s the share of the
row that is left."""
import math

import numpy as np
import pytest
import torch

import speculate_ref as ref
from test_gpu_verify import check, run

pytestmark = pytest.mark.gpu

MOST = np.float32(1.0 - 2.0 ** -24)         # the largest random number


def beside(border, distance):
    """The nearest fp32 numbers below and above a border that keep the distance."""
    lo, hi = np.float32(border - distance), np.float32(border + distance)
    while float(lo) > border - distance:
        lo = np.nextafter(lo, np.float32(0.0))
    while float(hi) < border + distance:
        hi = np.nextafter(hi, np.float32(2.0))
    return [u for u in (lo, hi) if 0.0 <= u < 1.0]


@pytest.mark.parametrize("V", [300, 5000, 50257])
@pytest.mark.parametrize("bits", [8, 14, 20, 22])
def test_fixed_drafts(V, bits):
    """The first child has all of p but 2^-bits of it; a second one, and the draw, from what is left."""
    rng = np.random.default_rng(V + bits)
    logits = rng.normal(size=V).astype(np.float32)
    first, second = V // 2, V // 3
    logits[second] = logits.max() + 2.0
    rest = np.delete(logits.astype(np.float64), first)
    logits[first] = np.float32(math.log(math.fsum(np.exp(rest))) + math.log(2.0 ** bits - 1.0))
    p = ref.softmax64(logits, 1.0)
    r = p.copy()
    r[first] = 0.0
    s = math.fsum(r)
    assert 2.0 ** -bits * 0.99 < s < 2.0 ** -bits * 1.01 and float(MOST) * math.fsum(p) >= p[first]
    distance = 1e-12 / s
    accept = beside(r[second] / s, distance)
    r2 = r.copy()
    r2[second] = 0.0
    # the draw, with and without the second child among the rejected
    draws = [u for w in (r, r2) for x in rng.choice(V - 2, 6) + 1
             for u in beside(math.fsum(w[:x]) / math.fsum(w), 1e-12 / math.fsum(w))]
    cases = [(MOST, u, d) for u in accept for d in (0.3, 0.8)] + [(MOST, MOST, d) for d in draws]
    B = len(cases)
    c = dict(logits=torch.from_numpy(logits).expand(3 * B, V).contiguous(), tokens=np.tile([0, first, second], B),
             parents=[[-1, 0, 0]] * B, u_accept=np.array([[0.5, a, b] for a, b, _ in cases], np.float32).reshape(-1),
             u_draw=np.array([d for *_, d in cases], np.float32))
    check(run(**c), **c)
    # one child alone: the draw from r without the first
    alone = dict(logits=c["logits"][:2 * B], tokens=np.tile([0, first], B), parents=[[-1, 0]] * B,
                 u_accept=np.full(2 * B, MOST), u_draw=c["u_draw"])
    check(run(**alone), **alone)


@pytest.mark.parametrize("V", [300, 5000, 50257])
@pytest.mark.parametrize("bits", [8, 14, 18])
def test_drawn_drafts(V, bits):
    """A drafting model within about 2^-bits of the target: what a rejection leaves is a difference of that size."""
    rng = np.random.default_rng(V + bits)
    logits = (rng.normal(size=V) * 2.0).astype(np.float32)
    p = ref.softmax64(logits, 1.0)
    q = (p * (1.0 + 2.0 ** -bits * rng.uniform(-1.0, 1.0, V))).astype(np.float32)
    left = np.maximum(p - q.astype(np.float64), 0.0)
    s = math.fsum(left)
    assert 2.0 ** -bits / 8 < s < 2.0 ** -bits
    distance = 1e-12 / s
    first = int(np.argmax(q.astype(np.float64) / p))
    assert float(MOST) * float(q[first]) >= p[first]
    border = left / s / q.astype(np.float64)
    seconds = [int(x) for x in rng.permutation(np.nonzero((border > 0.05) & (border < 0.95))[0])[:6]]
    assert len(seconds) == 6
    cases = [(x, u, d) for x in seconds for u in beside(border[x], distance) for d in (0.2, 0.7)]
    B = len(cases)
    c = dict(logits=torch.from_numpy(logits).expand(3 * B, V).contiguous(),
             tokens=np.array([[0, first, x] for x, *_ in cases]).reshape(-1), parents=[[-1, 0, 0]] * B,
             u_accept=np.array([[0.5, MOST, u] for _, u, _ in cases], np.float32).reshape(-1),
             u_draw=np.array([d for *_, d in cases], np.float32),
             probs=torch.from_numpy(q).expand(3 * B, V).contiguous())
    path, out, keep, lp = run(**c)
    # (the draws at 0.2 and 0.7 are not placed at borders: only the children are held here)
    want = [ref.verify(np.tile(logits.astype(np.float64), (3, 1)), [0, first, x], [-1, 0, 0], np.array([0.5, MOST, u]), d, 1.0,
                       np.tile(q.astype(np.float64), (3, 1)))[0] for x, u, d in cases]
    assert [row[:k].tolist() for row, k in zip(path, keep)] == want
    # the draw after one rejection
    up = np.cumsum(left)
    draws = [u for x in rng.choice(V - 2, 8) + 1 for u in beside(up[x - 1] / s, distance + 1e-12)]
    B = len(draws)
    d = dict(logits=c["logits"][:1].expand(2 * B, V).contiguous(), tokens=np.tile([0, first], B), parents=[[-1, 0]] * B,
             u_accept=np.full(2 * B, MOST), u_draw=np.array(draws, np.float32), probs=c["probs"][:1].expand(2 * B, V).contiguous())
    path, out, keep, lp = run(**d)
    for b, u in enumerate(draws):
        assert keep[b] == 1 and out[b, 0] == int(np.nonzero((up > float(u) * up[-1]) & (left > 0))[0][0]), (b, u)
