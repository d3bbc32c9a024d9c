"""Device plans that are not the planner's (GPU): a call ends, and touches
nothing beyond its tensors, whatever the plan holds.
"""
import pytest

pytestmark = pytest.mark.gpu

INT_MIN, INT_MAX = -(1 << 31), (1 << 31) - 1


@pytest.mark.parametrize("q,kv", [([90], [333]), ([200, 70], [333, 300]), ([300], [6500])])
@pytest.mark.parametrize("seen0", [INT_MIN, INT_MIN + 70, -(1 << 30)])
def test_rows_that_see_nothing_by_the_plan(q, kv, seen0):
    """A limit far below zero hides every key; it must not wrap into one far above."""
    import torch

    from test_gpu_prefill import Call
    c = Call(q, kv, 8, True, seed=31)
    good = c.plan.clone()
    items = c.plan[:8 * c.info.num_items].view(-1, 8)
    alone = items[:, 6] < 0                             # blocks whose keys are not split
    rows = torch.cat([torch.arange(r, r + n) for r, n in items[alone][:, :2].tolist()] or [torch.zeros(0, dtype=torch.long)]).cuda()
    items[:, 5] = seen0
    c.run()
    torch.cuda.synchronize()
    assert bool((c.out[rows] == 0.0).all()) and bool((c.lse[rows] == -float("inf")).all())
    c.plan.copy_(good)
    c.run()
    c.check("the planner's plan again")


@pytest.mark.parametrize("q_row", [INT_MAX, INT_MAX - 5, INT_MIN, 1 << 30])
def test_merges_of_rows_that_do_not_exist(q_row):
    """The merge's first row plus its rows may pass 2^31."""
    import torch

    from test_gpu_prefill import Call
    c = Call([60], [9000], 4, True, seed=32)
    assert c.info.num_merges == 1
    good = c.plan.clone()
    c.plan[8 * c.info.num_items] = q_row
    c.run()
    torch.cuda.synchronize()
    assert bool((c.out == 7.0).all()) and bool((c.lse == 7.0).all()), "rows that no merge belongs to"
    c.plan.copy_(good)
    c.run()
    c.check("the planner's plan again")
