"""What the prompt side's binding refuses by itself, before it asks for a device
(CPU only; no GPU work is launched).
"""
import os

import numpy as np
import pytest
import torch


@pytest.fixture(scope="module")
def mp():
    from paper_2609_36760_amd import _binding, _prefill
    if not os.path.exists(_binding.LIB_PATH):
        pytest.skip("libmla_lowbit.so not built (run __graft_entry__.build())")
    _prefill.library()
    return _prefill


def test_workspace_has_to_be_contiguous(mp):
    """A workspace whose elements share memory, or lie apart, holds fewer bytes than it has elements."""
    H = 2
    plan, info = mp.mla_plan_prefill([40], [5000], H)
    assert info.workspace_bytes > 0

    def rows(*shape):
        return torch.zeros(shape, dtype=torch.bfloat16)

    args = (info, torch.from_numpy(plan), rows(40, H, 128), rows(40, H, 64), rows(5000, H, 128), rows(5000, 64),
            rows(5000, H, 128), 0.07, rows(40, H, 128), torch.zeros(40, H))
    one = torch.zeros(1, dtype=torch.uint8)
    for bad in (one.expand(info.workspace_bytes), torch.zeros(2 * info.workspace_bytes, dtype=torch.uint8)[::2],
                torch.zeros(info.workspace_bytes // 4 // 128, 1).expand(-1, 128)):
        with pytest.raises(ValueError, match="workspace"):
            mp.mla_prefill_attn(*args, bad)


@pytest.mark.parametrize("bad", [np.array([2 ** 32 + 5]), np.array([-2 ** 32 + 5]), [3.7], [2 ** 31], [2 ** 70],
                                 torch.tensor([2 ** 33 + 1])])
def test_lengths_that_are_not_int32_are_refused(mp, bad):
    """A length that does not fit would otherwise wrap, or be cut, to another one and give a plan for that."""
    for at in range(4):
        lens = [[5], [9], None, None]
        lens[at] = bad
        with pytest.raises((ValueError, OverflowError)):
            mp.mla_plan_prefill(lens[0], lens[1], 2, True, lens[2], lens[3])


@pytest.mark.parametrize("kind", [list, tuple, np.array, torch.tensor, lambda x: np.array(x, np.int16), lambda x: np.array(x, np.uint32)])
def test_lengths_of_any_whole_type(mp, kind):
    want, _ = mp.mla_plan_prefill([5, 7], [9, 300], 2, True, [7, 0], [0, 0])
    got, info = mp.mla_plan_prefill(kind([5, 7]), kind([9, 300]), 2, True, kind([7, 0]), kind([0, 0]))
    assert np.array_equal(got, want) and (info.total_q, info.total_kv) == (12, 300)
    plan, info = mp.mla_plan_prefill(kind([]), kind([]), 2)
    assert plan.size == 0 and info.num_items == 0
    one, _ = mp.mla_plan_prefill(5, 9, 2)           # a number is a batch of one
    assert np.array_equal(one, mp.mla_plan_prefill([5], [9], 2)[0])
