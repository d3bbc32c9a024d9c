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
