"""The split size of tree calls whose node counts are given (CPU)."""
import math
import random

import pytest

from test_speculate_abi import EINVAL, mb, ms  # noqa: F401
from test_tree_split_estimate import estimate, looked_at


def lengths(seed, n, lo, hi):
    r = random.Random(seed)
    return [int(math.exp(r.uniform(math.log(lo), math.log(hi)))) for _ in range(n)]


def equal(n, k):
    return [k] * n


def ragged(n, k):
    r = random.Random(n + k)
    return [r.randrange(0, k + 1) for _ in range(n - 1)] + [k]


@pytest.mark.parametrize("trees", [equal, ragged])
@pytest.mark.parametrize("n,k,H,lo,hi", [(8, 4, 128, 1000, 32000), (24, 4, 128, 1000, 16000), (4, 16, 64, 8000, 128000),
                                         (21, 10, 16, 1000, 8000), (64, 4, 128, 1000, 32000), (70, 8, 16, 200, 4000),
                                         (32, 2, 32, 1000, 16000), (1, 7, 128, 5000, 5001), (24, 13, 64, 3000, 3020)])
def test_least_estimated_time(ms, n, k, H, lo, hi, trees):  # noqa: F811
    lens, nodes = lengths(n + k, n, lo, hi), trees(n, k)
    size = ms.mla_tree_split_tokens_for(lens, nodes, k, H)
    sizes = looked_at(lens, k, H)
    best = min(estimate(lens, nodes, H, k, s) for s in sizes)
    assert (size or sizes[0]) in sizes
    assert estimate(lens, nodes, H, k, size or sizes[0]) <= best * (1 + 1e-12)


@pytest.mark.parametrize("n,k,H,length,size", [(24, 13, 64, 3014, 2400), (8, 64, 16, 131136, 32800), (32, 8, 16, 4104, 544)])
def test_a_token_less_in_one_sequence_changes_nothing(ms, n, k, H, length, size):  # noqa: F811
    for lens in ([length] * n, [length] * (n - 1) + [length - 1], [length - 1] + [length] * (n - 1)):
        assert ms.mla_tree_split_tokens_for(lens, [k] * n, k, H) == size
    assert ms.mla_tree_split_tokens([length] * n, k, H) == size     # (sequences of one length are taken to be full)


def test_no_nodes_and_refusals(ms, mb):  # noqa: F811
    assert ms.mla_tree_split_tokens_for([], [], 4, 16) == 0
    assert ms.mla_tree_split_tokens_for([5000, 300], [0, 0], 4, 16) == 0
    assert ms.mla_tree_split_tokens_for([1], [0], 1, 1) == 0
    assert ms.mla_tree_split_tokens_for([2 ** 31 - 1] * 3, [1, 64, 0], 64, 16384) >= 0
    for bad in (([5], [-1], 4, 16), ([5], [5], 4, 16), ([0], [1], 4, 16), ([5], [1], 0, 16), ([5], [1], 65, 16), ([5], [1], 4, 0)):
        with pytest.raises(mb.MlaError):
            ms.mla_tree_split_tokens_for(*bad)
    for bad in (([5], [1, 2]), ([5, 6], [1]), ([[5]], [[1]]), ([5], [1.5]), ([5], [2 ** 31])):
        with pytest.raises((ValueError, OverflowError)):
            ms.mla_tree_split_tokens_for(*bad, 4, 16)
    lens = (5).to_bytes(4, "little")
    assert ms.library().mla_tree_split_tokens_for(lens, None, 1, 4, 16) == -EINVAL
    assert ms.library().mla_tree_split_tokens_for(None, lens, 1, 4, 16) == -EINVAL
    assert ms.library().mla_tree_split_tokens_for(None, None, 0, 4, 16) == 0
