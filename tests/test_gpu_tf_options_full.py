"""The transformer step with every option at the sizes that choose its largest
launches, against its oracle (bounds of tests/gpu_util.bf16_gate)."""
import pytest

from paper_2608_18469_amd import synth_tf
from tests.test_gpu_tf_options import ALL, _check
from tests.test_gpu_transformer import _bits_equal, _gpu_run, _trainer

pytestmark = pytest.mark.gpu


@pytest.mark.timeout(900)
def test_full_positions_match_oracle():
    """16 sequences of 1024 tokens, width 512: 256 partial rows of the layer norms'
    gradients (which Adam adds up in chunks of 32 elements) and both gradients of
    each block's packed projection in one launch of large tiles."""
    cfg = synth_tf.tf_config("tf_c5", vocab=512, layers=2, **ALL)
    params, batches = synth_tf.make_workload(cfg, seed=20, n_batches=1)
    tr = _trainer(cfg, params, keep_grads=False)
    tr.set_timing(True)
    tr.step(tr.device_tokens(batches[0]), "serial")
    tr.sync()
    pairs = [(r["tile_m"], r["tile_n"]) for r in tr.read_timing() if r["kind"] == "bwd_gemm" and r["layer"] == 0]
    tr.close()
    print("[tf options] full positions: launches of the projection's gradients", pairs, flush=True)
    assert len(pairs) == 2 and all(m >= 128 and n >= 128 for m, n in pairs), pairs
    _, gpu = _gpu_run(cfg, params, batches, "overlap")
    _, again = _gpu_run(cfg, params, batches, "serial")
    _bits_equal(gpu, again)
    print("[tf options] full positions: oracles", flush=True)
    _check(cfg, gpu, params, batches, "tf options, 16384 positions")


@pytest.mark.timeout(600)
@pytest.mark.parametrize("heads,layers,seq,batch", [(25, 2, 33, 3), (32, 2, 20, 2), (64, 1, 3, 2)])
def test_wide_models_match_oracle(heads, layers, seq, batch):
    """1600 and 2048 columns (four waves a row before the head) and 4096, the widest."""
    cfg = synth_tf.tf_config("tf_tiny", vocab=64, d=64 * heads, heads=heads, layers=layers, seq=seq, batch=batch, **ALL)
    params, batches = synth_tf.make_workload(cfg, seed=21, n_batches=1)
    print("[tf options] wide", heads, layers, seq, batch, flush=True)
    _, gpu = _gpu_run(cfg, params, batches, "overlap")
    _check(cfg, gpu, params, batches, "tf options, %d heads" % heads)
    _, again = _gpu_run(cfg, params, batches, "serial")
    _bits_equal(gpu, again)


@pytest.mark.parametrize("p", [2.0 ** -18, 1.0])
def test_extreme_dropout_matches_oracle(p):
    """Nothing dropped (p below half a step of 2^-16), and nothing kept."""
    cfg = synth_tf.tf_config("tf_small", **dict(ALL, dropout=p))
    params, batches = synth_tf.make_workload(cfg, seed=22, n_batches=1)
    print("[tf options] dropout", p, flush=True)
    _, gpu = _gpu_run(cfg, params, batches, "serial")
    _check(cfg, gpu, params, batches, "tf options, dropout %g" % p)
