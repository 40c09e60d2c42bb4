"""Refusals of the binding's gradient-row calls that no status of the library stands behind: nothing is launched."""
import pytest
import torch

from paper_2502_01703_b200 import binding as B


def _loss_inputs(T=4, width=64, vocab=10):
    return torch.zeros((T, width), dtype=torch.bfloat16), torch.zeros((vocab, width), dtype=torch.bfloat16), torch.zeros(T, dtype=torch.int64)


def test_a_strided_loss_is_refused():
    # the kernels write it as consecutive numbers
    with pytest.raises(ValueError, match="contiguous"):
        B.qless_lm_loss(*_loss_inputs(), out=dict(loss=torch.zeros(8)[::2]))
