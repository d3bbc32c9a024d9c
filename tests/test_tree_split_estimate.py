"""The split size of tree calls (CPU) has the least estimated time among the sizes that are
looked at, with the estimate written apart from the library's."""
import heapq

import pytest

from test_speculate_abi import mb, ms  # noqa: F401

CUS = 256


def estimate(lens, nodes, H, most, size):
    """us: workgroups of the row blocks of whole splits, then of the last ones, the longest first (past 64 sequences one
    sequence after the other), each on the compute unit that is free first; and the merge."""
    block = 64 if most * H <= 64 else 128
    fixed, tile = (18.5, 1.25) if block == 64 else (17.5, 1.6)
    whole, last, moved = [], [], 0
    for b, (length, n) in enumerate(zip(lens, nodes)):
        rows, full, left = n * H, length // size, length % size
        blocks = -(-rows // block)
        whole += [(b, 0, fixed + tile * (size // 32))] * (full * blocks)
        last += [(b, 1, fixed + tile * -(-left // 32))] * (blocks if left else 0)
        moved += rows * (full + bool(left)) if length > size else 0
    if len(lens) > 64:
        items = sorted(whole + last, key=lambda x: x[:2])
    else:
        items = whole + sorted(last, key=lambda x: -x[2])
    free, end = [0.0] * CUS, 0.0
    for *_, time in items:
        done = heapq.heappop(free) + time
        heapq.heappush(free, done)
        end = max(end, done)
    return end if not moved else end + 4.0 + 2.0 * moved * (512 * 2 + 8) / 4e6


def looked_at(lens, most, H):
    longest, block = max(lens), 64 if most * H <= 64 else 128
    size, sizes = 32, []
    while size < longest:
        sizes.append(size)
        size = -(-(size + max(size // 4, 1)) // 32) * 32
    sizes += [-(-longest // (parts * 32)) * 32 for parts in range(2, 33)]
    row_blocks = -(-most * H // block)
    return [-(-longest // 32) * 32] + [s for s in sizes if s < longest and (sum(lens) // s + len(lens)) * row_blocks <= 16 * CUS]


@pytest.mark.parametrize("k,H", [(4, 16), (13, 16), (4, 64), (2, 128), (9, 20)])
@pytest.mark.parametrize("n,length", [(1, 5000), (24, 3014), (64, 3000), (65, 3000), (70, 1100), (130, 2050), (200, 700)])
def test_sequences_of_one_length(ms, n, length, k, H):  # noqa: F811
    """Taken to have the most nodes each."""
    lens, nodes = [length] * n, [k] * n
    size, sizes = ms.mla_tree_split_tokens(lens, k, H), looked_at(lens, k, H)
    assert (size or sizes[0]) in sizes
    assert estimate(lens, nodes, H, k, size or sizes[0]) <= min(estimate(lens, nodes, H, k, s) for s in sizes) * (1 + 1e-12)
