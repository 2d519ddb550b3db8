"""Layer norms of rows far from zero: what the mean's own rounding may leave in
the output.  U = 2^-24 is the rounding of an fp32 operation
(tests/test_gpu_ops.py)."""
import numpy as np
import pytest

from oracle import ops_oracle as oo
from paper_2608_18469_amd import erase_ops as ops
from tests.test_gpu_ops import HALF, TINY, U, _dev, _np

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("C", [3, 33, 513, 700, 1025, 2049])
@pytest.mark.parametrize("value", [100.1, -7777.7, 30000.3, 1e6 + 0.3, 1.0 + 2.0 ** -23])
def test_rows_of_one_value_are_centred_to_zero(C, value):
    """Every output is the bias and every mean the value, exactly: in units of half
    the value's last place the first mean m is off by a whole number of at most
    2 C (1 + C u) (C roundings of at most 2 units each), so any partial sum of C
    differences x - m is a whole number below 2 C^2 (1 + C u) < 2^24 for C <= 2049,
    which fp32 adds without rounding; the mean of the differences is their value, which brings m to the
    value and each difference to 0."""
    import torch
    assert 2 * C * C * (1 + C * U) < 2 ** 24
    x = torch.full((5, C), value, device="cuda")
    w, b = torch.full((C,), 3.0, device="cuda"), torch.linspace(-1, 1, C, device="cuda")
    print("[norm, one value]", C, value, flush=True)
    y, m, r = ops.layer_norm(x, w, b)
    assert bool((m == x[:, 0]).all())
    assert torch.equal(y, b.expand(5, C))
    assert bool((r > 0).all()) and bool(torch.isfinite(r).all())


@pytest.mark.parametrize("C", [64, 401, 700, 1500, 2050, 4097, 9000, 16384])
@pytest.mark.parametrize("shift", [300.0, -1e4])
def test_rows_far_from_zero(C, shift):
    """The first mean is off by dm <= (C + 1) u mean|x|; x - m is exact (m is
    within a factor of 2 of x); the mean c of the differences by dc <= (C + 2) u
    (dm + mean|x - mean|), and that, with one rounding, is what is left in
    (x - m) - c."""
    import torch
    rng = np.random.Generator(np.random.PCG64(C))
    xa, x = _dev(rng.normal(size=(17, C)) + shift, "f32")
    w, wr = _dev(1 + 0.3 * rng.normal(size=C), "f32")
    b, br = _dev(rng.normal(size=C), "f32")
    print("[norm, far]", C, shift, flush=True)
    y, m, r = ops.layer_norm(xa, w, b)
    want, mean, rstd = oo.layer_norm(x, wr, br)
    d = np.abs(x - mean[:, None])
    dm = (C + 1) * U * np.abs(x).mean(1)
    assert (np.abs(x) > 2 * (d + dm[:, None])).all()  # so every difference is exact
    dc = (C + 2) * U * (dm + d.mean(1))
    assert (np.abs(_np(m) - mean) - (dc + U * np.abs(mean) * 1.01)).max() <= 0
    var = (d ** 2).mean(1)
    # mean of squares of x - m (its value var + the first mean's error squared), less c^2
    dv = (C + 4) * U * (var + dm ** 2) + 2 * dm * dc + dc ** 2
    dr = rstd * (0.5 * dv / (var + 1e-5) * 1.01 + 4 * U)
    assert (np.abs(_np(r) - rstd) - dr).max() <= 0
    h = d * rstd[:, None]
    dh = (dc[:, None] + U * d) * rstd[:, None] + h * (dr / rstd)[:, None] + U * h
    bound = dh * np.abs(wr) * 1.01 + 2 * U * (h * np.abs(wr) + np.abs(br)) + HALF["f32"] * np.abs(want)
    assert (np.abs(_np(y) - want) - bound).max() <= TINY


def test_statistics_of_bad_rows():
    """A NaN or infinity in a row shows in its statistics as in the formulas."""
    import torch
    x = torch.randn((4, 300), device="cuda")
    x[1, 5], x[2, 299], x[3, 0] = float("nan"), float("inf"), -float("inf")
    _, m, r = ops.layer_norm(x)
    assert bool(torch.isfinite(m[0])) and bool(torch.isnan(m[1])) and float(m[2]) == np.inf and float(m[3]) == -np.inf
    assert bool(torch.isfinite(r[0])) and bool(torch.isnan(r[1:]).all())
