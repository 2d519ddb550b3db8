"""The operators at places that only large tensors reach: dropout in several
launches, gradients stored beyond 32-bit offsets, long loops of rows."""
import numpy as np
import pytest

from oracle import ops_oracle as oo
from paper_2608_18469_amd import erase_ops as ops
from tests.test_gpu_ops import HALF, TINY, U, _norm_bounds, _np, _rope_case

pytestmark = pytest.mark.gpu


def test_dropout_in_two_launches():
    """2^30 + 5 rows of two groups of columns: a launch numbers 2^31 of them, the
    second one starts at row 2^30 (its x, residual and output, and the row that the
    generator counts)."""
    import torch
    R, C, p = (1 << 30) + 5, 9, 0.5
    x = torch.ones((R, C), dtype=torch.bfloat16, device="cuda")
    y = torch.full((R, C), 3.0, dtype=torch.bfloat16, device="cuda")
    at = [0, 1, (1 << 30) - 1, 1 << 30, (1 << 30) + 1, R - 1]
    x[at] = torch.arange(1, len(at) + 1, device="cuda")[:, None].bfloat16()
    y[at] = 16.0 * torch.arange(1, len(at) + 1, device="cuda")[:, None].bfloat16()
    print("[dropout] two launches", flush=True)
    ops.dropout(x, p, 77, 5, residual=y, out=y)
    for i, r in enumerate(at):
        kept = oo.dropout_kept(1, C, p, 77, 5, row0=r)[0][0]
        assert np.array_equal(_np(y[r]), 16.0 * (i + 1) + np.where(kept, 2.0 * (i + 1), 0.0)), r  # (exact in bf16)
    del y
    ops.dropout_backward(x, p, 77, 5, out=x)
    for i, r in enumerate(at):
        kept = oo.dropout_kept(1, C, p, 77, 5, row0=r)[0][0]
        assert np.array_equal(_np(x[r]), np.where(kept, 2.0 * (i + 1), 0.0)), r


@pytest.mark.parametrize("R", [1030, 700])
def test_layer_norm_gradients_beyond_32_bit_offsets(R):
    """Rows 2^23 elements apart: x, dy, res and dx beyond 2^32 elements, in two
    launches (1030 rows) and in one (700)."""
    import torch
    ld, C = 1 << 23, 96
    assert (R - 1) * ld > 1 << 32
    buf = torch.zeros(R * ld, dtype=torch.bfloat16, device="cuda")
    x, dy, res, dx = (buf.view(R, ld)[:, i * 128:i * 128 + C] for i in range(4))
    for t in (x, dy, res):
        t.copy_(torch.randn((R, C), device="cuda"))
    dx.fill_(7.0)
    w = torch.randn(C, device="cuda")
    xr, dr, rr, wr = _np(x), _np(dy), _np(res), _np(w)
    _, m, r = oo.layer_norm(xr)
    mean, rstd = torch.from_numpy(m).cuda().float(), torch.from_numpy(r).cuda().float()
    print("[norm backward, far rows]", R, flush=True)
    got = ops.layer_norm_backward(dy, x, w, mean, rstd, residual=res, out=(dx, None, None))
    mr, sr = _np(mean), _np(rstd)
    d64, w64, b64 = oo.layer_norm_backward(dr, xr, wr, mr, sr, rr)
    # the roundings of tests/test_gpu_ops.py, with |mean(g h)| bounded by the mean of |g h|
    h, g, n = np.abs(xr - mr[:, None]) * sr[:, None], np.abs(dr * wr), C + 2
    inner = g * 4 * U + (g.mean(1) * (n + 5) * U)[:, None] + h * ((g * h).mean(1) * (n + 11) * U)[:, None]
    bx = sr[:, None] * inner * 1.01 + 2 * U * np.abs(rr) + (HALF["bf16"] + U) * np.abs(d64)
    assert (np.abs(_np(dx) - d64) - bx).max() <= TINY
    assert (np.abs(_np(got[1]) - w64) - (R + 4) * U * (np.abs(dr) * h).sum(0)).max() <= TINY
    assert (np.abs(_np(got[2]) - b64) - (R + 1) * U * np.abs(dr).sum(0)).max() <= TINY
    buf.view(R, ld)[:, :512] = 0
    assert int(torch.count_nonzero(buf)) == 0  # nothing else was written


@pytest.mark.parametrize("dtype,C", [("bf16", 5), ("bf16", 129), ("f32", 600), ("bf16", 1600), ("f32", 9000)])
def test_layer_norm_rows_of_every_round(dtype, C):
    """More rows than the 2048 workgroups take in several rounds, the last round
    uneven: every row against the oracle."""
    import torch
    per = {5: 64, 129: 8, 600: 4, 1600: 1, 9000: 1}[C]  # rows a workgroup takes at once
    R = 2048 * per * 3 + per // 2 + 1
    x = torch.randn((R, C), device="cuda").to({"f32": torch.float32, "bf16": torch.bfloat16}[dtype])
    y, m, r = ops.layer_norm(x)
    print("[norm, rounds]", dtype, R, C, flush=True)
    for i in range(0, R, 1 << 14):
        s = slice(i, min(R, i + (1 << 14)))
        xr = _np(x[s])
        want, wm, wr = oo.layer_norm(xr)
        by, bm, br = _norm_bounds(xr, None, None, wm, wr, want, dtype, C, 1e-5)
        assert (np.abs(_np(y[s]) - want) - by).max() <= TINY
        assert (np.abs(_np(m[s]) - wm) - bm).max() <= TINY and (np.abs(_np(r[s]) - wr) - br).max() <= TINY


def test_layer_norm_of_the_most_rows():
    """2^31 - 1 rows of one column: y is the bias, the mean the value."""
    import torch
    R = (1 << 31) - 1
    x = torch.empty((R, 1), dtype=torch.bfloat16, device="cuda").normal_()
    b = torch.full((1,), 0.375, device="cuda")
    mean = torch.full((R,), float("nan"), device="cuda")
    print("[norm, most rows]", flush=True)
    y, m, _ = ops.layer_norm(x, None, b, out=(torch.zeros_like(x), mean, None))
    for i in range(0, R, 1 << 28):
        s = slice(i, min(R, i + (1 << 28)))
        assert bool((m[s] == x[s, 0]).all()) and bool((y[s] == 0.375).all())


@pytest.mark.parametrize("dtype,layout,Hq,Hk,D,rot", [("bf16", "half", 1100, 40, 64, 64), ("f32", "interleaved", 600, 1, 80, 48),
                                                      ("bf16", "interleaved", 4096, 4096, 8, 2), ("f32", "half", 5, 300, 1024, 1024)])
def test_rope_of_many_heads(dtype, layout, Hq, Hk, D, rot):
    """The heads of one token over several workgroups."""
    _rope_case(dtype, layout, 1, 3, Hq, Hk, D, dict(rot_dim=rot), "far")
    _rope_case(dtype, layout, 2, 1, Hq, Hk, D, dict(rot_dim=rot), "none", start=7, inplace=True, backward=True)
