"""Commit over so many layers and sequences that a workgroup takes several layers, the
last one fewer (GPU), byte for byte."""
import numpy as np
import pytest
import torch

import speculate_ref as ref
from test_gpu_commit import commit, padded, random_caches

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("kind", ref.KINDS)
@pytest.mark.parametrize("B,layers", [(40, 25), (60, 47), (513, 2), (600, 5)])
def test_several_layers_of_a_workgroup(kind, B, layers):
    """2 of 25 layers each, 6 of 47, 3 of 2 and 6 of 5: with a last group of 1, 5, 2 and 5."""
    rng = np.random.default_rng(B)
    most = 9
    ctx = rng.integers(0, 60, B).tolist()
    paths = [[0] + sorted(rng.choice(np.arange(1, most), int(rng.integers(0, most - 1)), replace=False).tolist()) for _ in range(B)]
    table, num_pages = ref.block_table(rng, [c + most for c in ctx], 32)
    caches = random_caches(B, layers, num_pages * ref.page_bytes(kind, 32))
    before = np.stack([c.cpu().numpy() for c in caches])
    keep = [len(p) for p in paths]
    lens = commit(kind, caches, 32, table, num_pages, ctx, padded(paths, most), keep)
    want, want_lens = ref.commit(before, kind, 32, table, num_pages, ctx, padded(paths, most), keep, most)
    assert np.array_equal(np.stack([c.cpu().numpy() for c in caches]), want)
    assert lens.tolist() == want_lens.tolist()
