"""The transformer step with options (rotary positions, layer norms, dropout)
against its oracle (oracle/tf_options_oracle.py), at the bounds of the plain
step (tests/gpu_util.bf16_gate); schedules, resumed runs and steps without
options next to it."""
import numpy as np
import pytest

from oracle import tf_options_oracle as too
from paper_2608_18469_amd import synth_tf
from tests.gpu_util import bf16_gate
from tests.test_gpu_transformer import _bits_equal, _gpu_run, _trainer, _worst

pytestmark = pytest.mark.gpu

ROPE = dict(rope=dict(rot_dim=64))
PART = dict(rope=dict(rot_dim=24, layout="interleaved", scaling="by_parts", factor=4.0, original_length=64.0))
NORM = dict(norm="layer")
DROP = dict(dropout=0.2, dropout_seed=(1 << 63) + 12345)
ALL = dict(ROPE, **NORM, **DROP)


def _oracle(cfg, params, batches, emulate_bf16=False, dtype=np.float64):
    m, v, p, t, recs = synth_tf.zero_state(params), synth_tf.zero_state(params), params, 0, []
    for tok in batches:
        r = too.tf_step(cfg, p, m, v, t, tok, emulate_bf16=emulate_bf16, dtype=dtype)
        p, m, v, t = r["params"], r["m"], r["v"], r["t"]
        pk = lambda tree: [synth_tf.pack_block(cfg, b, tree[b]) for b in range(cfg["layers"])]
        recs.append({"losses": np.array(r["losses"]), "params": pk(p), "m": pk(m), "v": pk(v), "grads": pk(r["grads"])})
    return recs


def _check(cfg, gpu, params, batches, label):
    r64, rbf = _oracle(cfg, params, batches), _oracle(cfg, params, batches, emulate_bf16=True)
    rbf32 = _oracle(cfg, params, batches, emulate_bf16=True, dtype=np.float32) if len(batches) > 1 else None
    return bf16_gate(lambda a, b: _worst(cfg, a, b), gpu, r64, rbf, rbf32, label=label)


@pytest.mark.parametrize("name,opts", [("rope", ROPE), ("rope part", PART), ("norm", NORM), ("dropout", DROP), ("all", ALL),
                                       ("all part", dict(PART, **NORM, norm_eps=1e-3, dropout=0.5))])
def test_small_two_steps_match_oracle(name, opts):
    cfg = synth_tf.tf_config("tf_small", **opts)
    params, batches = synth_tf.make_workload(cfg, seed=5, n_batches=2)
    print("[tf options]", name, flush=True)
    _, gpu = _gpu_run(cfg, params, batches, "serial")
    _check(cfg, gpu, params, batches, "tf " + name)
    _, again = _gpu_run(cfg, params, batches, "overlap")
    _bits_equal(gpu, again)


@pytest.mark.parametrize("vocab,heads,layers,seq,batch", [
    (64, 1, 2, 1, 1), (64, 1, 2, 16, 2), (512, 3, 2, 65, 3), (512, 2, 3, 256, 2), (128, 8, 2, 40, 2), (64, 16, 2, 9, 3),
    (64, 22, 2, 17, 2), (64, 33, 2, 8, 2), (4160, 2, 2, 64, 2), (2112, 2, 2, 700, 2)])
def test_shapes_match_oracle(vocab, heads, layers, seq, batch):
    """Widths of every row shape, ragged positions, the wide logits (multiples of
    256) and the head's gradient in slices; one step with everything on."""
    cfg = synth_tf.tf_config("tf_tiny", vocab=vocab, d=64 * heads, heads=heads, layers=layers, seq=seq, batch=batch, **ALL)
    params, batches = synth_tf.make_workload(cfg, seed=6, n_batches=1)
    print("[tf options]", vocab, heads, layers, seq, batch, flush=True)
    _, gpu = _gpu_run(cfg, params, batches, "overlap")
    _check(cfg, gpu, params, batches, "tf %d heads" % heads)
    _, again = _gpu_run(cfg, params, batches, "serial")
    _bits_equal(gpu, again)


def test_a_resumed_run_draws_the_masks_of_an_uninterrupted_one():
    cfg = synth_tf.tf_config("tf_small", **ALL)
    params, batches = synth_tf.make_workload(cfg, seed=7, n_batches=3)
    _, whole = _gpu_run(cfg, params, batches)
    tr, first = _gpu_run(cfg, params, batches[:1])
    tree = lambda flats: [synth_tf.unpack_block(cfg, b, f) for b, f in enumerate(flats)]
    p, m, v, _g = tr.flat_state()
    tr.close()
    tr = _trainer(cfg, tree(p), m=tree(m), v=tree(v), step=1)
    _, rest = _gpu_run(cfg, params, batches[1:], tr=tr)
    _bits_equal(whole, first + rest)
    # and another seed draws others
    other = dict(cfg, dropout_seed=1)
    _, got = _gpu_run(other, params, batches[:1])
    assert not np.array_equal(got[0]["grads"][0], whole[0]["grads"][0])


def test_a_rotation_by_no_angle_changes_nothing():
    """Sequences of one token (position 0) give the plain step's results bit for
    bit through the rotation's launches."""
    cfg = synth_tf.tf_config("tf_small", seq=1)
    params, batches = synth_tf.make_workload(cfg, seed=8, n_batches=2)
    _, plain = _gpu_run(cfg, params, batches)
    _, same = _gpu_run(dict(cfg, **ROPE), params, batches)  # position 0 alone: angle 0
    _bits_equal(plain, same)


def test_without_kept_gradients_and_beside_another_context():
    """No gradient buffers, and a plain trainer stepping in between: same numbers."""
    cfg = synth_tf.tf_config("tf_small", **ALL)
    params, batches = synth_tf.make_workload(cfg, seed=10, n_batches=2)
    _, want = _gpu_run(cfg, params, batches)
    plain = synth_tf.tf_config("tf_small")
    pp, pb = synth_tf.make_workload(plain, seed=11, n_batches=1)
    other = _trainer(plain, pp)
    tr = _trainer(cfg, params, keep_grads=False)
    for tok in batches:
        t, o = tr.device_tokens(tok), other.device_tokens(pb[0])
        tr.step(t, "overlap")
        other.step(o, "overlap")
    tr.sync()
    other.sync()
    p, m, v, g = tr.flat_state()
    assert all(x is None for x in g)
    for got, ref in ((p, want[-1]["params"]), (m, want[-1]["m"]), (v, want[-1]["v"])):
        assert all(np.array_equal(a, b) for a, b in zip(got, ref))
    tr.close()
    other.close()


def test_a_token_out_of_range_is_reported():
    from paper_2608_18469_amd import erase
    cfg = synth_tf.tf_config("tf_tiny", **ALL)
    params, batches = synth_tf.make_workload(cfg, seed=12, n_batches=1)
    tok = batches[0].copy()
    tok[0, 3] = cfg["vocab"]
    tr = _trainer(cfg, params)
    tr.step(tr.device_tokens(tok), "serial")
    with pytest.raises(erase.EraseError) as e:
        tr.sync()
    assert e.value.status == erase.ERR_INVALID_ARG
    tr.close()


def test_timing_records_with_options():
    cfg = synth_tf.tf_config("tf_small", **ALL)
    params, batches = synth_tf.make_workload(cfg, seed=9, n_batches=1)
    tr = _trainer(cfg, params)
    t = tr.device_tokens(batches[0])
    tr.set_timing(True)
    tr.step(t, "overlap")
    tr.sync()
    kinds = [r["kind"] for r in tr.read_timing()]
    tr.close()
    L = cfg["layers"]
    assert kinds.count("rope") == 2 * L and kinds.count("dropout") == 4 * L
    assert kinds.count("rms_fwd") == 3 * L and kinds.count("rms_bwd") == 3 * L
    assert all(r in ("prologue", "empty") or kinds.count(r) >= 1 for r in kinds)
