"""New lengths of a commit right beside the memory that it reads (GPU)."""
import numpy as np
import pytest
import torch

import speculate_ref as ref
from test_gpu_commit import random_caches

pytestmark = pytest.mark.gpu
DEV = "cuda"


def test_new_lengths_beside_the_inputs():
    from paper_2609_36760_amd import _speculate as ms
    rng = np.random.default_rng(3)
    table, num_pages = ref.block_table(rng, [50, 90], 64)
    caches = random_caches(1, 2, num_pages * ref.page_bytes("c4"))
    ints = torch.tensor([0, 0, 40, 80, 2, 3, 0, 0, 0, 2, 0, 0, 4, 5, 0, 0], dtype=torch.int32, device=DEV)
    args = dict(ctx_lens=ints[2:4], keep=ints[4:6], path=ints[8:14].view(2, 3))
    for at in (0, 6, 14):
        ms.mla_lowbit_commit(ref.library_format("c4"), ms.layer_caches(caches), num_pages, torch.from_numpy(table).to(DEV),
                             new_lens=ints[at:at + 2], **args)
        assert ints[at:at + 2].tolist() == [42, 83]
