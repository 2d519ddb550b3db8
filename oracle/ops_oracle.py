"""CPU oracle of the transformer operators: rotary positions, layer norm and
dropout, forward and backward, from their definitions in float64.

TEST INFRASTRUCTURE ONLY.  Nothing in the product path imports, links or runs
this module: only the test-suite does.  It shares no code with the HIP library.
"""
from __future__ import annotations

import numpy as np

__all__ = ["rope_frequencies", "rope", "rope_backward", "layer_norm", "layer_norm_backward", "philox", "dropout_kept",
           "dropout", "dropout_backward"]


def rope_frequencies(rot_dim, base=10000.0, scaling="none", factor=1.0, original_length=0.0, fast=32.0, slow=1.0):
    """(f [rot_dim / 2], amplitude): angle per position of every pair."""
    i = np.arange(rot_dim // 2, dtype=np.float64)
    g = base ** (-2.0 * i / rot_dim)
    if scaling == "none":
        return g, 1.0
    if scaling == "linear":
        return g / factor, 1.0
    if scaling == "ntk":  # the slowest pair ends up interpolated by the factor, the fastest unchanged
        last = max(1, rot_dim // 2 - 1)
        return g * factor ** (-i / last), 1.0
    keep = np.clip((original_length * g / (2 * np.pi) - slow) / (fast - slow), 0.0, 1.0)
    return g * (keep + (1 - keep) / factor), 0.1 * np.log(factor) + 1.0


def rope(x, positions, freq, amplitude=1.0, layout="half", sign=1.0):
    """x [B][T][H][D], positions [B][T]: pairs of the first 2 len(freq) columns
    times amplitude exp(i sign p f)."""
    x = np.array(x, dtype=np.float64)
    n = len(freq)
    z = amplitude * np.exp(1j * sign * np.asarray(positions, np.float64)[:, :, None, None] * np.asarray(freq))
    at = (slice(0, n), slice(n, 2 * n)) if layout == "half" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    w = (x[..., at[0]] + 1j * x[..., at[1]]) * z
    x[..., at[0]], x[..., at[1]] = w.real, w.imag
    return x


def rope_backward(dy, positions, freq, amplitude=1.0, layout="half"):
    """The transposed map: the gradient at x of <dy, rope(x)>."""
    return rope(dy, positions, freq, amplitude, layout, sign=-1.0)


def layer_norm(x, w=None, b=None, eps=1e-5):
    """(y, mean, rstd) of every row."""
    x = np.asarray(x, np.float64)
    m = x.mean(1)
    r = 1.0 / np.sqrt(((x - m[:, None]) ** 2).mean(1) + eps)
    y = (x - m[:, None]) * r[:, None]
    if w is not None:
        y = y * np.asarray(w, np.float64)
    if b is not None:
        y = y + np.asarray(b, np.float64)
    return y, m, r


def layer_norm_backward(dy, x, w, mean, rstd, res=None):
    """(dx, dw, db) from the forward's statistics."""
    dy, x = np.asarray(dy, np.float64), np.asarray(x, np.float64)
    r = np.asarray(rstd, np.float64)[:, None]
    h = (x - np.asarray(mean, np.float64)[:, None]) * r
    g = dy if w is None else dy * np.asarray(w, np.float64)
    dx = r * (g - g.mean(1, keepdims=True) - h * (g * h).mean(1, keepdims=True))
    if res is not None:
        dx = dx + np.asarray(res, np.float64)
    return dx, (dy * h).sum(0), dy.sum(0)


def philox(counter, key, rounds=10):
    """Philox4x32 (Salmon, Moraes, Dror, Shaw 2011): counter [..., 4] and key (2)
    of 32-bit words -> [..., 4]."""
    c = [np.asarray(counter[..., i], np.uint64) for i in range(4)]
    low, by = np.uint64(0xFFFFFFFF), np.uint64(32)
    for i in range(rounds):
        k = [np.uint64((int(key[j]) + i * w) & 0xFFFFFFFF) for j, w in enumerate((0x9E3779B9, 0xBB67AE85))]
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> by) ^ c[1] ^ k[0], b & low, (a >> by) ^ c[3] ^ k[1], a & low]
    return np.stack(c, -1).astype(np.uint32)


def dropout_kept(rows, cols, p, seed, offset, row0=0):
    """(kept [rows][cols], scale): column c of row r takes half c % 8 of the
    words of counter (c / 8, r, offset)."""
    limit = int(np.floor(p * 65536 + 0.5))
    groups = -(-cols // 8)
    counter = np.zeros((rows, groups, 4), np.uint64)
    counter[..., 0] = np.arange(groups)
    counter[..., 1] = (row0 + np.arange(rows))[:, None]
    counter[..., 2], counter[..., 3] = offset & 0xFFFFFFFF, offset >> 32
    words = philox(counter, (seed & 0xFFFFFFFF, seed >> 32))
    halves = np.stack([words & np.uint32(0xFFFF), words >> np.uint32(16)], -1).reshape(rows, 8 * groups)[:, :cols]
    return halves >= limit, 65536.0 / (65536 - limit) if limit < 65536 else 0.0


def dropout(x, p, seed, offset=0, res=None):
    x = np.asarray(x, np.float64)
    kept, scale = dropout_kept(*x.shape, p, seed, offset)
    y = np.where(kept, x, 0.0) * scale
    return y if res is None else y + np.asarray(res, np.float64)


def dropout_backward(dy, p, seed, offset=0):
    return dropout(dy, p, seed, offset)
