"""Expanded attention on very large and very small values (GPU): finite inputs
give finite outputs, whatever weights the values meet on the way -- scores that
grow by tens of units behind a row's first keys, many keys of equal weight,
blocks done over, and partials that are merged.
"""
import math

import numpy as np
import pytest

from unseen_keys import check_finite_case

pytestmark = pytest.mark.gpu

TAU32 = float(np.float32(1.0 / math.sqrt(192.0)))       # as a call takes it
SHAPES = [([200], [1500]), ([90], [700]), ([1], [64]), ([3], [5000]), ([257], [3000]), ([1, 2, 1], [3000, 70, 4099])]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("grow", [0.0, 10.0, 31.0, 60.0, 200.0, -35.0, -80.0])
@pytest.mark.parametrize("top", [2.0 ** 126, 2.0 ** 84, 2.0 ** -40])
@pytest.mark.parametrize("q,kv", SHAPES)
def test_values_far_from_one(q, kv, causal, grow, top):
    import torch

    from test_gpu_prefill import TAU, Call
    c = Call(q, kv, 2, causal, seed=21)
    g = torch.Generator(device="cuda")
    g.manual_seed(22)
    # head 0: values of either sign; head 1: of one sign, so that nothing cancels
    c.v[:] = ((torch.rand(c.v.shape, generator=g, device="cuda") * 1.98 - 0.99) * top).bfloat16()
    c.v[:, 1] = c.v[:, 1].abs()
    # all keys but the first 40 of each sequence stand `grow` above those (40: a tile's edge is at 32 and 64)
    c.q_nope[:, :, 0] = 32.0
    c.k_nope[:, :, 0] = grow / (TAU * 32.0)
    for e in c.k0:
        c.k_nope[e:e + 40, :, 0] = 0.0
    c.run()
    check_finite_case(c, range(2), f"{q} on {kv}, values to {top:.3g}, grown by {grow}")


@pytest.mark.parametrize("q,kv", [([128], [770]), ([250], [1537])])
@pytest.mark.parametrize("top", [2.0 ** 126, 2.0 ** -40])
def test_values_far_from_one_under_equal_weights(q, kv, top):
    """All scores 0: a row's sum is its number of keys."""
    from test_gpu_prefill import Call
    c = Call(q, kv, 2, True, seed=23)
    c.q_nope[:], c.q_rope[:] = 0.0, 0.0
    c.v[:, 0] = top
    c.v[:, 1] = -top
    c.run()
    check_finite_case(c, range(2), f"{q} on {kv}, all values {top:.3g}")


@pytest.mark.parametrize("q,kv,causal", [([200], [1500], True), ([90], [700], True), ([1], [64], True), ([128], [770], True),
                                         ([256], [8200], True), ([70, 3], [70, 5000], False)])
@pytest.mark.parametrize("which", ["first", "every third", "last", "first 100"])
def test_seen_keys_that_score_minus_infinity(q, kv, causal, which):
    """They weigh nothing, and what the others give is exact to the usual roundings."""
    from test_gpu_prefill import Call
    c = Call(q, kv, 2, causal, seed=24)
    c.q_nope[:, :, 0] = c.q_nope[:, :, 0].abs() + 0.5
    for e, nk in zip(c.k0, kv):
        k = c.k_nope[e:e + nk, :, 0]
        at = {"first": slice(0, 1), "every third": slice(0, nk, 3), "last": slice(nk - 1, nk), "first 100": slice(0, min(100, nk - 1))}[which]
        k[at] = -float("inf")
    c.run()
    check_some_rows(c, f"{q} on {kv}, {which} at -inf")


def check_some_rows(c, what):
    """check_finite_case without the causal rows whose keys all score -inf (their output is not a number)."""
    import torch
    torch.cuda.synchronize()
    for b, (nq, nk) in enumerate(zip(c.q_lens, c.kv_lens)):
        a, e = c.q0[b], c.k0[b]
        finite = torch.isfinite(c.k_nope[e:e + nk, 0, 0])
        for i in range(nq):
            sees = nk - nq + i + 1 if c.causal else nk
            if sees > 0 and not finite[:sees].any():
                assert bool(c.out[a + i].isnan().all()) and bool((c.lse[a + i] == -float("inf")).all())
                c.out[a + i] = 0.0
    check_finite_case(c, range(2), what)


@pytest.mark.parametrize("q,kv", [([1], [1]), ([64], [64]), ([200], [300]), ([3], [5000]), ([257], [3000])])
@pytest.mark.parametrize("grow", [0.0, 60.0])
def test_lse_keeps_32_bits(q, kv, grow):
    """Scores that are exact in fp32: lse is as near to the formula's as fp32 takes it, beside references too.

    k is 0 but in one channel of 0 or 1, q in that channel a multiple of 1/8: the products are exact.  In units of 2^-24:
    softmax_scale log2(e) is off by 2 and the score's difference from the reference rounds by 1, together at most 4 |z|;
    exp2 2; the sum 1 for every step of the longest chain (16 in a key block, one per key block, one for the halves); the
    logarithm 2 and the last sum and product 2, of lse; merging adds 2 for a weight and one per partial (the chains' room
    for it: splits have at least 4 key blocks)."""
    import torch

    from test_gpu_prefill import TAU, Call
    c = Call(q, kv, 2, True, seed=25)
    for t in (c.q_nope, c.q_rope, c.k_nope, c.k_rope):
        t[:] = 0.0
    g = torch.Generator(device="cuda")
    g.manual_seed(26)
    nq, nk = q[0], kv[0]
    c.q_nope[:nq, :, 0] = torch.randint(1, 16, (nq, 2), generator=g, device="cuda").bfloat16() / 8.0
    c.k_nope[:nk, :, 0] = torch.randint(0, 2, (nk, 2), generator=g, device="cuda").bfloat16()
    if grow:                                            # all but the first 40 keys, by 74: the rows are done over
        c.q_nope[:nq, :, 1] = 8.0
        c.k_nope[40:nk, :, 1] = 128.0
    c.run()
    torch.cuda.synchronize()
    for h in range(2):
        z = TAU32 * (c.q_nope[:nq, h].double() @ c.k_nope[:nk, h].double().T.contiguous())
        hidden = torch.arange(nk, device="cuda")[None] >= (torch.arange(nq, device="cuda") + nk - nq + 1)[:, None]
        lse = torch.logsumexp(z.masked_fill(hidden, -float("inf")), 1)
        size = z.masked_fill(hidden, 0.0).abs().amax(1)
        bound = 2.0 ** -24 * (4.0 * size + 2.0 + 17.0 + nk / 32.0 + 4.0 * lse.abs() + 2.0)
        r = float(((c.lse[:nq, h].double() - lse).abs() / bound).max())
        print(f"  {q} on {kv}, {grow}: lse off by {r:.2f} of its bound", flush=True)
        assert r <= 1.0
