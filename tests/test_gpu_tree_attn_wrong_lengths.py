"""A context length that fits nothing (GPU): only its own sequence's rows are affected,
in batches of up to 64 sequences, whose launch adds lengths up, and in larger ones."""
import pytest
import torch

from test_gpu_tree_attn import Batch, trees

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("split", [0, 64])
@pytest.mark.parametrize("n", [3, 64, 70])
def test_other_sequences_keep_their_rows(n, split):
    ctx = [(37 * i) % 300 for i in range(n)]
    b = Batch(91, "c4", 16, ctx, trees(13, [1 + i % 6 for i in range(n)]), behind=1)
    plan = b.plan(split)
    b.call(**plan)
    b.check(split)
    out, lse = b.out.clone(), b.lse.clone()
    for at in (0, 1, n - 1):
        others = torch.ones(b.T, dtype=torch.bool, device=out.device)
        others[int(b.cu[at]):int(b.cu[at + 1])] = False
        for length in (2 ** 31 - 1, 2 ** 31 - 6, 1 << 30, -(2 ** 31), -1):
            print("sequence", at, "length", length, flush=True)
            b.ctx_d[at] = length
            b.out.fill_(-77.0)
            b.lse.fill_(-77.0)
            if plan:
                plan["workspace"].fill_(255)
            b.call(**plan)
            assert torch.equal(b.out[others].view(torch.int16), out[others].view(torch.int16)), (at, length)
            assert torch.equal(b.lse[others], lse[others]), (at, length)
        b.ctx_d[at] = ctx[at]
