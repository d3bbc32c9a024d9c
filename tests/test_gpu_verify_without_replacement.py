"""Siblings drawn without replacement (GPU): given as fixed drafts, the emitted tokens are
distributed as the target's."""
import numpy as np
import pytest
import torch

from test_gpu_verify import run

pytestmark = pytest.mark.gpu


def test_given_as_fixed_drafts_they_leave_the_target_alone():
    """40 000 sequences, three children drawn without replacement from a q far from p; each frequency within 5
    deviations of its own, as for six tokens one of 3.5e6 runs would fail by chance."""
    V, B = 6, 40000
    rng = np.random.default_rng(5)
    logits = torch.tensor(rng.normal(size=(1, V)) * 1.5, dtype=torch.float32)
    p = torch.softmax(logits.double(), 1)[0].numpy()
    q = rng.dirichlet(np.ones(V))
    order = np.argsort(np.log(q)[None] - np.log(rng.exponential(size=(B, V))), axis=1)[:, ::-1]     # drawn one after the other
    tokens = np.concatenate([np.zeros((B, 1), np.int64), order[:, :3]], 1)
    c = dict(logits=logits.expand(4 * B, V).contiguous(), tokens=tokens.reshape(-1), parents=[[-1, 0, 0, 0]] * B,
             u_accept=rng.random(4 * B, np.float32), u_draw=rng.random(B, np.float32))
    path, out, keep, lp = run(**c)
    got = np.bincount(out[:, 0], minlength=V) / B
    assert np.all(np.abs(got - p) <= 5 * np.sqrt(p * (1 - p) / B)), (got, p)
