"""Host-only checks of the transformer step's options: sizes, parameter counts
and refusals (no GPU needed)."""
import ctypes

import pytest

from paper_2608_18469_amd import erase, erase_tf, synth_tf

INVALID, SHAPE = erase.ERR_INVALID_ARG, erase.ERR_SHAPE
ALL = dict(rope=dict(rot_dim=64), norm="layer", dropout=0.1, dropout_seed=3)


@pytest.mark.parametrize("opts", [dict(), dict(norm="layer"), dict(rope=dict(rot_dim=64)), ALL])
def test_param_count_and_roundtrip(opts):
    import numpy as np
    cfg = synth_tf.tf_config("tf_tiny", **opts)
    params, _ = synth_tf.make_workload(cfg)
    for b in range(cfg["layers"]):
        n = erase_tf.param_count(cfg, b)
        assert n == synth_tf.param_count(cfg, b)
        flat = synth_tf.pack_block(cfg, b, params[b])
        assert flat.size == n
        back = synth_tf.unpack_block(cfg, b, flat)
        assert all(np.array_equal(back[k], params[b][k]) for k in params[b])
    plain = erase_tf.param_count(synth_tf.tf_config("tf_tiny"), 1)
    assert erase_tf.param_count(cfg, 1) - plain == (6 * cfg["d"] if opts.get("norm") == "layer" else 0)


def test_no_options_are_the_plain_step():
    cfg = synth_tf.tf_config("tf_small")
    assert erase_tf.native_options(cfg) is None
    L, nc, n, p = erase_tf.lib(), erase_tf.native_config(cfg), ctypes.c_size_t(0), ctypes.c_size_t(0)
    assert L.erase_tf_workspace_bytes(ctypes.byref(nc), ctypes.byref(n)) == 0
    assert L.erase_tf_workspace_bytes_options(ctypes.byref(nc), None, ctypes.byref(p)) == 0
    assert n.value == p.value
    zero = erase_tf.TfOptions()
    assert L.erase_tf_workspace_bytes_options(ctypes.byref(nc), ctypes.byref(zero), ctypes.byref(p)) == 0
    assert n.value == p.value
    assert erase_tf.workspace_bytes(dict(cfg, **ALL)) > n.value


def _options(**kw):
    o = erase_tf.native_options(synth_tf.tf_config("tf_small", **ALL))
    for k, v in kw.items():
        setattr(o.rope_spec if k in ("rot_dim", "scaling", "base", "factor") else o, k, v)
    return o


@pytest.mark.parametrize("kw,code", [
    (dict(rope=2), INVALID), (dict(rope=-1), INVALID), (dict(rope_layout=2), INVALID), (dict(rot_dim=66), SHAPE),
    (dict(rot_dim=3), SHAPE), (dict(rot_dim=0), SHAPE), (dict(scaling=9), INVALID), (dict(base=0.0), INVALID),
    (dict(scaling=1, factor=0.0), INVALID), (dict(norm=2), INVALID), (dict(norm_eps=-1.0), INVALID),
    (dict(norm_eps=float("nan")), INVALID), (dict(dropout=-0.1), INVALID), (dict(dropout=1.5), INVALID),
    (dict(dropout=float("nan")), INVALID)])
def test_bad_options(kw, code):
    cfg = synth_tf.tf_config("tf_small")
    L, nc, o = erase_tf.lib(), erase_tf.native_config(cfg), _options(**kw)
    n, c, ctx = ctypes.c_size_t(0), ctypes.c_int64(0), ctypes.c_void_p()
    assert L.erase_tf_workspace_bytes_options(ctypes.byref(nc), ctypes.byref(o), ctypes.byref(n)) == code
    assert L.erase_tf_param_count_options(ctypes.byref(nc), ctypes.byref(o), 0, ctypes.byref(c)) == code
    bufs = (erase.BlockBuffers * cfg["layers"])(*[erase.BlockBuffers(0x1000, 0x2000, 0x3000, None)] * cfg["layers"])
    assert L.erase_tf_init_options(ctypes.byref(nc), ctypes.byref(o), bufs, 0x100000, 1 << 40, 0x10, 0x20,
                                   ctypes.byref(ctx)) == code
    assert ctx.value is None


def test_options_that_are_off_are_not_read():
    cfg = synth_tf.tf_config("tf_small")
    L, nc, n = erase_tf.lib(), erase_tf.native_config(cfg), ctypes.c_size_t(0)
    for kw in (dict(rope=0, rot_dim=3, rope_layout=7), dict(norm=0, norm_eps=float("nan"))):
        o = _options(**kw)
        assert L.erase_tf_workspace_bytes_options(ctypes.byref(nc), ctypes.byref(o), ctypes.byref(n)) == 0


def test_a_workspace_for_the_plain_step_is_too_small():
    cfg = synth_tf.tf_config("tf_tiny")
    L, nc, o, ctx = erase_tf.lib(), erase_tf.native_config(cfg), _options(), ctypes.c_void_p()
    need = erase_tf.workspace_bytes(cfg)
    bufs = (erase.BlockBuffers * 2)(*[erase.BlockBuffers(0x1000, 0x2000, 0x3000, None)] * 2)
    assert L.erase_tf_init_options(ctypes.byref(nc), ctypes.byref(o), bufs, 0x100000, need, 0x10, 0x20,
                                   ctypes.byref(ctx)) == erase.ERR_WORKSPACE
