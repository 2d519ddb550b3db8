"""Pins of the transformer oracle with options: without options it is
transformer_oracle's step, rotations make scores depend on distances, masks
drop what they say, and the gradients of the added parts agree with central
differences."""
import numpy as np
import pytest

from oracle import ops_oracle as oo, tf_options_oracle as too, transformer_oracle as to
from paper_2608_18469_amd import synth_tf

OPTS = dict(rope=dict(rot_dim=32, layout="interleaved", scaling="by_parts", factor=4.0, original_length=64.0), norm="layer",
            norm_eps=1e-4, dropout=0.3, dropout_seed=77)


def _workload(**kw):
    cfg = synth_tf.tf_config("tf_tiny", seq=7, **kw)
    params, toks = synth_tf.make_workload(cfg, 3, 1)
    return cfg, params, synth_tf.zero_state(params), toks[0]


def test_without_options_it_is_the_plain_step():
    cfg, params, zero, tok = _workload()
    a, b = too.tf_step(cfg, params, zero, zero, 4, tok), to.tf_step(cfg, params, zero, zero, 4, tok)
    assert np.allclose(a["losses"], b["losses"], rtol=1e-13)
    for name in ("grads", "params", "m", "v"):
        for x, y in zip(a[name], b[name]):
            for k in x:
                assert np.allclose(x[k], y[k], rtol=1e-9, atol=1e-13), (name, k)


@pytest.mark.parametrize("which", ["rope", "norm", "dropout", "all"])
def test_gradients_by_differences(which):
    opts = OPTS if which == "all" else {k: v for k, v in OPTS.items() if k.split("_")[0] == which}
    cfg, params, zero, tok = _workload(**opts)
    r = too.tf_step(cfg, params, zero, zero, 0, tok)
    rng = np.random.Generator(np.random.PCG64(1))
    for b in range(cfg["layers"]):
        for k, x in params[b].items():
            dirn = rng.normal(size=x.shape)
            e = 1e-5
            moved = []
            for sgn in (1, -1):
                q = [dict(p) for p in params]
                q[b][k] = np.asarray(x, np.float64) + sgn * e * dirn
                moved.append(too.tf_step(cfg, q, zero, zero, 0, tok)["losses"][b])
            got = float((r["grads"][b][k] * dirn).sum())
            want = (moved[0] - moved[1]) / (2 * e)
            assert abs(got - want) <= 1e-6 * max(1.0, abs(want)), (b, k, got, want)


def test_dropout_of_everything_leaves_the_residual_stream():
    cfg, params, zero, tok = _workload(dropout=1.0)
    r = too.tf_step(cfg, params, zero, zero, 0, tok)
    for b in range(cfg["layers"]):
        assert all(not r["grads"][b][k].any() for k in ("wqkv", "wo", "w1", "w2"))
    # every block's head sees the embedding rows alone
    a0 = np.asarray(params[0]["emb"], np.float64)[tok[:, :-1].reshape(-1)]
    hn = a0 / np.sqrt((a0 * a0).mean(1, keepdims=True) + 1e-6)
    for b in range(cfg["layers"]):
        rows, _ = to.softmax_xent(hn @ np.asarray(params[b]["wh"], np.float64).T, tok[:, 1:].reshape(-1))
        assert abs(rows.mean() - r["losses"][b]) < 1e-12


def test_masks_differ_by_step_block_and_branch():
    seen = [oo.dropout_kept(14, 64, 0.5, 77, (s << 40) + t)[0] for s in range(4) for t in (1, 2)]
    for i in range(len(seen)):
        for j in range(i):
            assert (seen[i] != seen[j]).mean() > 0.3
