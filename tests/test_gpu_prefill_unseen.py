"""Expanded attention where keys are split: rows that see nothing of a split
beside rows of their wave that do (GPU).

Their scores on the split's keys, which they do not see, are far above those
on the keys that they see, or infinite; the rows that see these keys score
ordinarily on them, so nothing asks for the rows to be done over.
"""
import pytest

from unseen_keys import check_finite_case, split_edges

pytestmark = pytest.mark.gpu

SHAPES = [(128, 770, 1), (128, 770, 16), (100, 800, 2), (250, 1537, 2), (256, 8200, 16), (169, 12559, 16)]


@pytest.mark.parametrize("gap", [40, 110, 160, 400, float("inf")])
@pytest.mark.parametrize("q,kv,H", SHAPES)
def test_unseen_keys_of_a_split_have_no_part(q, kv, H, gap):
    from test_gpu_prefill import TAU, Call
    c = Call([q], [kv], H, True, seed=q + kv)
    edges = split_edges(c.plan.cpu().numpy(), c.info)
    assert edges, "the plan has no split that some rows of a wave see nothing of"
    c.q_nope[:q, :, 0] = -1.0 if gap == float("inf") else 0.0
    c.k_nope[:kv, :, 0] = 0.0
    for q_row, rows, key0, blind in edges:
        c.k_nope[key0 + 1, :, 0] = 64.0 if gap < 1e30 else gap      # among the split's first 32 keys
        c.q_nope[q_row:q_row + len(blind), :, 0] = 32.0 if gap == float("inf") else gap / (TAU * 64.0)
    c.run()
    check_finite_case(c, range(min(H, 3)), f"{q} rows on {kv} keys, {H} heads, unseen by {gap}")
