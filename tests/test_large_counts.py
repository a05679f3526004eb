"""Counts that 32 bits do not hold reach the library as what no call takes, not cut
to their last 32 bits (argument checks only; nothing is enqueued, so no GPU is needed)."""
import os

import pytest
import torch

BF, F32 = torch.bfloat16, torch.float32
MANY = 2**32 + 3


@pytest.fixture()
def steps(monkeypatch):
    """The binding with tensors of this machine taken for the current device's."""
    from paper_2609_10264_amd import _lib
    from paper_2609_10264_amd import steps
    if not os.path.exists(_lib.LIB_PATH):
        pytest.skip("libmvk.so not built (run __graft_entry__.build())")
    monkeypatch.setattr(steps, "_where", lambda stream: (-1, 0))
    return steps


def _refused(call):
    from paper_2609_10264_amd import MvkError, _lib
    with pytest.raises(MvkError) as e:
        call()
    assert e.value.status == _lib.MVK_ERANGE, e.value


def test_block_norm(steps):
    x, y, h = (torch.zeros((1, 1)).expand(MANY, 1) for _ in range(3))
    _refused(lambda: steps.block_norm(x, out=y, residual_out=h))
    x, y, h = (torch.empty((1, MANY), dtype=BF) for _ in range(3))  # (never touched)
    _refused(lambda: steps.block_norm(x, out=y, residual_out=h))


def test_gated_activation(steps):
    g, u, y = (torch.zeros((1, 1)).expand(MANY, 1) for _ in range(3))
    _refused(lambda: steps.gated_activation(g, u, out=y))
    g, u, y = (torch.empty((1, MANY), dtype=BF) for _ in range(3))
    _refused(lambda: steps.gated_activation(g, u, out=y))


def test_sample(steps):
    x, u, out = torch.empty((1, MANY), dtype=BF), torch.zeros(1), torch.zeros(1, dtype=torch.int32)
    _refused(lambda: steps.sample(x, u, out=out))
    x, u, out = torch.zeros((1, 1)).expand(MANY, 1), torch.empty(MANY), torch.empty(MANY, dtype=torch.int32)
    _refused(lambda: steps.sample(x, u, out=out))
