"""Attention of drafted tokens for queries that are not finite, or past the fp16 range
over a low-bit cache (GPU): the same results unsplit, with few splits and with many."""
import math

import numpy as np
import pytest
import torch

import speculate_ref as ref
from test_gpu_tree_attn import Batch, trees

pytestmark = pytest.mark.gpu

# (contexts, nodes, split): unsplit; sequences of one split among others; so many splits that the merge shares a row
# between waves; more sequences than lanes
FORMS = [([150, 20, 33], 0), ([150, 20, 33], 64), ([1100, 900, 1500], 32), ([130, 40, 0, 75, 200] * 14, 64)]


@pytest.mark.parametrize("ctx,split", FORMS, ids=["unsplit", "few", "many", "70_sequences"])
@pytest.mark.parametrize("kind,H", [("c4", 8), ("c2p", 20), ("bf16", 16)])
def test_rows_of_queries_that_are_not_finite(kind, H, ctx, split):
    """Rows with a NaN or an infinity among their queries are NaN, all others as ever."""
    b = Batch(81, kind, H, ctx, trees(11, [6] * len(ctx)), behind=1)
    rows = [(1, 0, 7, math.nan), (2, H - 1, 540, math.nan), (6, 1, 300, math.inf), (9, 3, 575, -math.inf), (11, 2, 0, math.nan)]
    for node, head, channel, value in rows:
        b.q[node, head, channel] = value
        (b.q_lat[node, head] if channel < 512 else b.q_rope[node, head])[channel % 512] = value
        b.q[node, head, channel] = math.nan         # what is expected of the row
    b.call(**b.plan(split))
    print("of the bound:", b.check(split))
    for node, head, *_ in rows:
        assert b.out[node, head].isnan().all() and b.lse[node, head].isnan()


@pytest.mark.parametrize("ctx,split", FORMS, ids=["unsplit", "few", "many", "70_sequences"])
@pytest.mark.parametrize("kind", ["c4", "c2p"])
def test_rows_of_queries_past_the_fp16_range(kind, ctx, split):
    """A query channel that becomes an infinity as an fp16 operand: scores are infinities by the sign of the key's
    channel.  One that is +inf makes the row NaN; a row of -inf alone weighs no key."""
    H, nodes = 8, [6] * len(ctx)
    strange = {}
    for s, n in enumerate(c + k for c, k in zip(ctx, nodes)):
        for t in range(n):
            def put(row):
                row[64:128] = torch.linspace(3.0, 5.0, 64)          # one sign, not 0 when dequantized
            strange[(s, t)] = put
    b = Batch(82, kind, H, ctx, trees(12, nodes), strange=strange)
    up, down = [(1, 0), (8, 3)], [(2, 1), (7, 5)]
    for rows, value in ((up, 1e6), (down, -1e6)):
        for node, head in rows:
            b.q[node, head, 100] = value
            b.q_lat[node, head, 100] = value
    b.call(**b.plan(split))
    torch.cuda.synchronize()
    cache = b.cache.cpu().numpy()
    for s in range(2):
        x = ref.cached_values(cache, kind, b.table[s], b.lens[s])
        assert (x[:, 100] > 0.5).all() and np.isfinite(x).all()
    for node, head in up:
        assert b.out[node, head].isnan().all() and b.lse[node, head].isnan()
    for node, head in down:
        assert (b.out[node, head] == 0).all() and b.lse[node, head] == -math.inf
        b.out[node, head] = math.nan                                # (out of the check of all other rows)
        b.lse[node, head] = math.nan
    for node, head in up + down:
        b.q[node, head, 100] = math.nan
    b.check(split)
