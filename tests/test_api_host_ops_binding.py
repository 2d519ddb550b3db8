"""Calls of the operators' binding (erase_ops, erase_tf options) that it refuses
by itself, before any memory is read or any HIP call is made (no GPU needed)."""
import pytest
import torch

from paper_2608_18469_amd import erase, erase_ops as ops

INVALID, SHAPE = erase.ERR_INVALID_ARG, erase.ERR_SHAPE


@pytest.mark.parametrize("device", ["cpu", torch.device("cpu"), torch.device("meta")])
def test_a_table_lives_on_a_gpu(device):
    with pytest.raises(erase.EraseError) as e:
        ops.rope_table(64, device=device)
    assert e.value.status == INVALID
