"""Pins of the operators' oracle against definitions that do not use it:
torch's layer_norm and its autograd, complex rotations by scalar arithmetic,
the scalings' limits, published Philox4x32-10 outputs, central differences of
every gradient."""
import math

import numpy as np
import pytest
import torch

from oracle import ops_oracle as oo


def _rng(seed):
    return np.random.Generator(np.random.PCG64(seed))


def test_philox_known_answers():
    """The known answers that accompany the paper's generator (all-zero, all-one and digits-of-pi inputs)."""
    f = 0xFFFFFFFF
    for ctr, key, want in (
            ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
            ((f, f, f, f), (f, f), (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
            ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0),
             (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1))):
        assert tuple(int(v) for v in oo.philox(np.array([ctr], np.uint64), key)[0]) == want


def test_dropout_share_and_scale():
    kept, scale = oo.dropout_kept(256, 513, 0.3, 5, 9)
    limit = round(0.3 * 65536)
    n = kept.size
    # six standard deviations of a binomial share
    assert abs(kept.mean() - (1 - limit / 65536)) <= 6 * math.sqrt(0.3 * 0.7 / n)
    assert scale * (65536 - limit) == 65536
    assert oo.dropout_kept(3, 9, 0.0, 1, 2)[0].all() and not oo.dropout_kept(3, 9, 1.0, 1, 2)[0].any()
    other, _ = oo.dropout_kept(256, 513, 0.3, 5, 10)
    assert abs((kept == other).mean() - (0.3 ** 2 + 0.7 ** 2)) <= 6 * 0.5 / math.sqrt(n)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rope_is_a_rotation_by_scalars(layout):
    rng = _rng(1)
    x = rng.normal(size=(2, 3, 2, 10))
    pos = np.array([[0, -4, 100000], [7, 7, 1]])
    f, a = oo.rope_frequencies(6)
    y = oo.rope(x, pos, f, a, layout)
    for b in range(2):
        for t in range(3):
            for h in range(2):
                for i in range(3):
                    i1, i2 = (i, i + 3) if layout == "half" else (2 * i, 2 * i + 1)
                    th = float(pos[b, t]) * 10000.0 ** (-2 * i / 6)
                    x1, x2 = x[b, t, h, i1], x[b, t, h, i2]
                    assert abs(y[b, t, h, i1] - (x1 * math.cos(th) - x2 * math.sin(th))) < 1e-10
                    assert abs(y[b, t, h, i2] - (x2 * math.cos(th) + x1 * math.sin(th))) < 1e-10
                assert np.array_equal(y[b, t, h, 6:], x[b, t, h, 6:])
    # scores depend on the distance alone
    q, k = rng.normal(size=(1, 1, 1, 10)), rng.normal(size=(1, 1, 1, 10))
    s = [float((oo.rope(q, [[p + 5]], f)[..., :6] * oo.rope(k, [[p]], f)[..., :6]).sum()) for p in (0, 123)]
    assert abs(s[0] - s[1]) < 1e-11


def test_rope_scalings():
    f, _ = oo.rope_frequencies(64)
    assert np.allclose(oo.rope_frequencies(64, scaling="linear", factor=4)[0], f / 4, rtol=1e-15)
    n, _ = oo.rope_frequencies(64, scaling="ntk", factor=4)
    assert n[0] == f[0] and abs(n[-1] / f[-1] - 0.25) < 1e-12
    assert np.allclose(n, (10000 * 4 ** (64 / 62)) ** (-2 * np.arange(32) / 64), rtol=1e-13)
    p, a = oo.rope_frequencies(64, scaling="by_parts", factor=4, original_length=4096)
    turns = 4096 * f / (2 * np.pi)
    assert np.allclose(p[turns >= 32], f[turns >= 32], rtol=1e-15) and np.allclose(p[turns <= 1], f[turns <= 1] / 4, rtol=1e-15)
    assert (turns >= 32).any() and (turns <= 1).any() and ((turns > 1) & (turns < 32)).any()
    assert abs(a - (1 + 0.1 * math.log(4))) < 1e-15
    for s in ("linear", "ntk", "by_parts"):
        g, a = oo.rope_frequencies(64, scaling=s, factor=1.0, original_length=4096)
        assert np.allclose(g, f, rtol=1e-15) and a == 1.0


def _differences(f, x, dy, eps=1e-6):
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        p, m = x.copy(), x.copy()
        p[i] += eps
        m[i] -= eps
        g[i] = ((f(p) - f(m)) * dy).sum() / (2 * eps)
    return g


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rope_backward_by_differences(layout):
    rng = _rng(2)
    x, dy = rng.normal(size=(1, 2, 2, 6)), rng.normal(size=(1, 2, 2, 6))
    f, a = oo.rope_frequencies(4, scaling="by_parts", factor=8, original_length=64)
    pos = np.array([[3, 500]])
    g = oo.rope_backward(dy, pos, f, a, layout)
    assert np.allclose(g, _differences(lambda v: oo.rope(v, pos, f, a, layout), x, dy), atol=1e-8)


def test_layer_norm_against_torch_and_differences():
    rng = _rng(3)
    x, dy, res = (rng.normal(size=(4, 7)) + 3.0 for _ in range(3))
    w, b = rng.normal(size=7), rng.normal(size=7)
    y, m, r = oo.layer_norm(x, w, b, 1e-3)
    tx, tw, tb = (torch.from_numpy(v).requires_grad_() for v in (x, w, b))
    ty = torch.nn.functional.layer_norm(tx, (7,), tw, tb, 1e-3)
    assert np.allclose(y, ty.detach().numpy(), atol=1e-12)
    ty.backward(torch.from_numpy(dy))
    dx, dw, db = oo.layer_norm_backward(dy, x, w, m, r, res)
    assert np.allclose(dx - res, tx.grad.numpy(), atol=1e-12)
    assert np.allclose(dw, tw.grad.numpy(), atol=1e-12) and np.allclose(db, tb.grad.numpy(), atol=1e-12)
    assert np.allclose(dx - res, _differences(lambda v: oo.layer_norm(v, w, b, 1e-3)[0], x, dy), atol=1e-7)
    assert np.allclose(dw, _differences(lambda v: oo.layer_norm(x, v, b, 1e-3)[0], w, dy), atol=1e-7)
    # without weight and bias: ones and zeros
    assert np.array_equal(oo.layer_norm(x)[0], oo.layer_norm(x, np.ones(7), np.zeros(7))[0])
    assert np.array_equal(oo.layer_norm_backward(dy, x, None, m, r)[0], oo.layer_norm_backward(dy, x, np.ones(7), m, r)[0])


def test_dropout_backward_by_differences():
    rng = _rng(4)
    x, dy, res = (rng.normal(size=(3, 11)) for _ in range(3))
    g = oo.dropout_backward(dy, 0.4, 77, 3)
    assert np.allclose(g, _differences(lambda v: oo.dropout(v, 0.4, 77, 3, res), x, dy), atol=1e-8)
