"""Angles of the rotary tables against 60-digit arithmetic, and of positions up
to the furthest that a call takes."""
import decimal
import math
from decimal import Decimal

import numpy as np
import pytest

from paper_2608_18469_amd import erase_ops as ops
from tests.test_gpu_ops import TINY, U, _dev, _np

pytestmark = pytest.mark.gpu

TAU = 2 * Decimal("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899")
SPECS = [dict(rot_dim=64), dict(rot_dim=2), dict(rot_dim=128, base=500000.0), dict(rot_dim=1024), dict(rot_dim=48, base=1.0),
         dict(rot_dim=96, base=1e300), dict(rot_dim=40, scaling="linear", factor=3.0), dict(rot_dim=128, scaling="ntk", factor=8.0),
         dict(rot_dim=64, scaling="by_parts", factor=8.0, original_length=4096.0),
         dict(rot_dim=64, scaling="by_parts", factor=1.7, original_length=100.0)]


def _turns(rot_dim, base=10000.0, scaling="none", factor=1.0, original_length=0.0, fast=32.0, slow=1.0):
    """f_i / (2 pi) to about 60 digits."""
    with decimal.localcontext() as c:
        c.prec = 70
        b, s, r = Decimal(base), Decimal(factor), Decimal(rot_dim)
        if scaling == "ntk":
            b *= (s.ln() * r / (r - 2)).exp()
        out = []
        for i in range(rot_dim // 2):
            g = (b.ln() * (-2 * i) / r).exp()
            if scaling == "linear":
                g /= s
            if scaling == "by_parts":
                k = (Decimal(original_length) * g / TAU - Decimal(slow)) / (Decimal(fast) - Decimal(slow))
                k = min(Decimal(1), max(Decimal(0), k))
                g *= k + (1 - k) / s
            out.append(g / TAU)
        return out


@pytest.mark.parametrize("spec", SPECS)
def test_table_against_exact_arithmetic(spec):
    """Within 2^-63 turns a position: the power's rounded exponent (f ln(1 / f) <=
    1 / e of 2^-64), the power, the scaling and the quotient (a few roundings of
    2^-64), all times 1 / (2 pi), and half a unit of 2^-64 for the fraction."""
    words = ops.rope_table(**spec).data.cpu().numpy().astype(np.uint64)
    want = _turns(**spec)
    assert len(words) == len(want) + 1
    with decimal.localcontext() as c:
        c.prec = 70
        one = Decimal(2) ** 64
        off = [abs(Decimal(int(a)) - t * one) for a, t in zip(words, want)]
        assert max(off) <= 2, float(max(off))


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("spec", SPECS)
@pytest.mark.parametrize("start", [0, (1 << 31) - 3, -(1 << 31), (1 << 40) - 1, -(1 << 40)])
def test_positions_of_every_distance(spec, layout, start):
    """The angle is off by |p| 2^-63 turns of the table and 2^-32 that the kernel
    drops; the rest is 10 roundings of |x1| + |x2| (tests/test_gpu_ops.py)."""
    n, T = spec["rot_dim"] // 2, 3
    rng = np.random.Generator(np.random.PCG64(n))
    x, ref = _dev(rng.normal(size=(1, T, 1, 2 * n)), "f32")
    print("[rope, far]", spec, layout, start, flush=True)
    y, _ = ops.rope(x, None, ops.rope_table(**spec), start=start, layout=layout)
    amp = 0.1 * math.log(spec["factor"]) + 1 if spec.get("scaling") == "by_parts" else 1.0
    with decimal.localcontext() as c:
        c.prec = 70
        f = _turns(**spec)
        angle = np.array([[float((t * (start + p)) % 1 * TAU) for t in f] for p in range(T)])
    x1, x2 = (ref[0, :, 0, :n], ref[0, :, 0, n:]) if layout == "half" else (ref[0, :, 0, ::2], ref[0, :, 0, 1::2])
    got = _np(y)[0, :, 0]
    y1, y2 = (got[:, :n], got[:, n:]) if layout == "half" else (got[:, ::2], got[:, 1::2])
    cs, sn = np.cos(angle), np.sin(angle)
    far = 2 * np.pi * ((abs(start) + T) * 2.0 ** -63 + 2.0 ** -32)
    bound = amp * (np.abs(x1) + np.abs(x2)) * (10 * U + far) + TINY
    for got, want in ((y1, amp * (x1 * cs - x2 * sn)), (y2, amp * (x2 * cs + x1 * sn))):
        assert (np.abs(got - want) - bound - U * np.abs(want)).max() <= 0


def test_a_table_filled_on_a_busy_stream():
    """A stream that the caller orders after the filling one reads a filled table,
    with no synchronisation of the host in between."""
    import torch
    x = torch.randn((2, 300, 4, 64), device="cuda")
    want, _ = ops.rope(x, None, ops.rope_table(64, base=777.0))
    fill, use = torch.cuda.Stream(), torch.cuda.Stream()
    big = torch.randn((4096, 4096), device="cuda")
    torch.cuda.synchronize()
    got, tables = [], []
    for _ in range(3):
        with torch.cuda.stream(fill):
            for _ in range(20):  # a few milliseconds before the fill
                big @ big
        table = ops.rope_table(64, base=777.0, stream=fill)
        use.wait_stream(fill)
        tables.append(table)  # (its memory is the filling stream's)
        got.append(ops.rope(x, None, table, stream=use)[0])
    torch.cuda.synchronize()
    assert all(torch.equal(y, want) for y in got)
