"""Calls of the operators' binding (erase_ops, erase_tf options) that it refuses
by itself, before any memory is read or any HIP call is made (no GPU needed)."""
import pytest
import torch

from paper_2608_18469_amd import erase, erase_ops as ops, erase_tf, synth_tf

INVALID, SHAPE = erase.ERR_INVALID_ARG, erase.ERR_SHAPE


@pytest.mark.parametrize("device", ["cpu", torch.device("cpu"), torch.device("meta")])
def test_a_table_lives_on_a_gpu(device):
    with pytest.raises(erase.EraseError) as e:
        ops.rope_table(64, device=device)
    assert e.value.status == INVALID


def test_a_table_holds_its_pairs():
    """Memory that is shorter than its rotation, or of another kind: a call would
    read behind it."""
    spec = ops.RopeSpec(64, 0, 10000.0, 1.0, 0.0, 32.0, 1.0)
    assert ops.RopeTable(spec, torch.zeros(33, dtype=torch.int64)).rot_dim == 64
    for data in (torch.zeros(32, dtype=torch.int64), torch.zeros(0, dtype=torch.int64), torch.zeros(33, dtype=torch.int32),
                 torch.zeros(33, dtype=torch.float64), torch.zeros(66, dtype=torch.int64)[::2],
                 torch.zeros(1, dtype=torch.int64).expand(33)):
        with pytest.raises(erase.EraseError) as e:
            ops.RopeTable(spec, data)
        assert e.value.status == INVALID


@pytest.mark.parametrize("opts", [
    dict(norm="batch"), dict(norm=None), dict(rope=dict(rot_dim=64, layout="both")), dict(rope=dict(rot_dim=64, scaling="cubic")),
    dict(rope=dict()), dict(rope=dict(base=500000.0))])
def test_unknown_names_of_step_options(opts):
    cfg = synth_tf.tf_config("tf_tiny", **opts)
    for call in (lambda: erase_tf.native_options(cfg), lambda: erase_tf.param_count(cfg, 0), lambda: erase_tf.workspace_bytes(cfg)):
        with pytest.raises(erase.EraseError) as e:
            call()
        assert e.value.status == INVALID


@pytest.mark.parametrize("rot_dim", [(1 << 32) + 64, 1 << 31, (1 << 31) - 2, -(1 << 32) + 64, 1 << 64])
def test_rotations_beyond_32_bits_are_not_taken_modulo(rot_dim):
    for call in (lambda: ops.rope_table(rot_dim), lambda: ops.rope_frequencies(rot_dim),
                 lambda: erase_tf.workspace_bytes(synth_tf.tf_config("tf_tiny", rope=dict(rot_dim=rot_dim)))):
        with pytest.raises(erase.EraseError) as e:
            call()
        assert e.value.status == SHAPE

