"""New lengths of a commit that share memory with what it reads (CPU): refused, by the C
entry points for the lengths and counts, by the binding for the paths."""
import pytest
import torch

from test_speculate_abi import COMMIT, EINVAL, mb, ms, status  # noqa: F401


@pytest.mark.parametrize("name", ["mla_lowbit_commit", "mla_bf16_commit"])
def test_entry_points(ms, mb, name):  # noqa: F811
    base = dict(COMMIT, fmt=mb.cache_format(), ctx_lens=4096, keep=8192, path=256, B=5)
    for at in (4096, 4096 + 16, 4096 - 16, 8192, 8192 + 16, 8192 - 16):
        assert status(ms, name, base, dict(new_lens=at)) == EINVAL, at


@pytest.mark.parametrize("low", [True, False])
def test_binding(ms, mb, low):  # noqa: F811
    whole = torch.zeros(1 << 17, dtype=torch.uint8)
    at = -whole.data_ptr() % 256
    fmt = mb.cache_format()
    size = mb.mla_lowbit_page_bytes(fmt) if low else mb.mla_bf16_page_bytes(fmt)
    layers = ms.layer_caches([whole[at:at + size]])
    ints = torch.zeros(64, dtype=torch.int32)
    args = dict(num_pages=1, block_table=torch.zeros((4, 3), dtype=torch.int32), ctx_lens=ints[0:4], keep=ints[8:12],
                path=ints[16:36].view(4, 5), new_lens=None)
    call = ms.mla_lowbit_commit if low else ms.mla_bf16_commit
    for first in (13, 16, 20, 35):
        with pytest.raises(ValueError, match="memory of its own"):
            call(fmt, layers, **dict(args, new_lens=ints[first:first + 4]))
