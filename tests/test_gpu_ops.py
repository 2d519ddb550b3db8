"""The transformer operators (include/erase_ops.h) on the GPU against the float64
oracle (oracle/ops_oracle.py), at the sizes, strides, types and values where
they can go wrong.

Tolerances count roundings: u = 2^-24 for each fp32 operation and half a step
of the output's type (2^-8 bf16, 2^-24 fp32) for the one final rounding.  The
sums' bounds hold for every order of n additions: (n - 1) u times the sum of
magnitudes."""
import numpy as np
import pytest

from oracle import ops_oracle as oo
from paper_2608_18469_amd import erase, erase_ops as ops

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
TINY = 1e-37  # below the smallest normal numbers (flushed or not)


def _t(dtype):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]


def _dev(a, dtype):
    """The array in `dtype` on the GPU, and its float64 values."""
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda().to(_t(dtype))
    return t, t.double().cpu().numpy()


def _np(t):
    return t.double().cpu().numpy()


def _inside(t, lead, ld):
    """t [rows][cols] again inside a larger buffer, `lead` elements from its start, with pitch ld: (view, buffer)."""
    import torch
    R, C = t.shape
    buf = torch.full((lead + max(R, 1) * ld + 8,), 7.0, dtype=t.dtype, device="cuda")
    v = buf[lead:lead + R * ld].view(R, ld)[:, :C]
    v.copy_(t)
    return v, buf


def _rest_untouched(buf, lead, R, C, ld):
    b = buf.clone()
    b[lead:lead + R * ld].view(R, ld)[:, :C] = 7.0
    return bool((b == 7.0).all())


# ---------------------------------------------------------------------------
# rotary positions
# ---------------------------------------------------------------------------
def _check_rope(y, x, pos, spec, layout, sign, dtype, what):
    f, a = oo.rope_frequencies(**spec)
    want = oo.rope(x, pos, f, a, layout, sign)
    n = len(f)
    at = (slice(0, n), slice(n, 2 * n)) if layout == "half" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    # cos and sin: 3 roundings of an angle below pi / 4, 2 of the polynomial, 2 of
    # the amplitude; 2 of the products and the sum: 10 u of |x1| + |x2|.  The
    # oracle's own angle p f has 2 roundings of double at its size.
    mag = (np.abs(x[..., at[0]]) + np.abs(x[..., at[1]])) * a
    angle = np.abs(np.asarray(pos, np.float64))[:, :, None, None] * f
    bound = np.zeros_like(want)
    bound[..., at[0]] = bound[..., at[1]] = mag * (10 * U + angle * 2.0 ** -51)
    bound[..., :2 * n] += HALF[dtype] * np.abs(want[..., :2 * n])
    err = np.abs(y - want) - bound
    assert err.max() <= TINY, (what, float(err.max()))


def _rope_case(dtype, layout, B, T, Hq, Hk, D, spec, positions, start=0, lay="bthd", lead=0, inplace=False, backward=False,
               seed=0):
    import torch
    what = (dtype, layout, B, T, Hq, Hk, D, spec, positions, start, lay, lead, inplace, backward)
    print("[rope]", what, flush=True)
    rng = np.random.Generator(np.random.PCG64(seed + B * 1000 + T * 10 + D))

    def make(H):
        x, ref = _dev(rng.normal(size=(B, T, H, D)), dtype)
        if lay == "bthd":
            buf = torch.full((lead + x.numel() + 8,), 7.0, dtype=x.dtype, device="cuda")
            v = buf[lead:lead + x.numel()].view(B, T, H, D)
        elif lay == "bhtd":
            buf = torch.full((lead + x.numel() + 8,), 7.0, dtype=x.dtype, device="cuda")
            v = buf[lead:lead + x.numel()].view(B, H, T, D).transpose(1, 2)
        else:  # columns of a wider row, with a gap behind every head
            buf = torch.full((lead + B * T * H * (D + 3) + 8,), 7.0, dtype=x.dtype, device="cuda")
            v = buf[lead:lead + B * T * H * (D + 3)].view(B, T, H, D + 3)[..., :D]
        v.copy_(x)
        return v, ref, buf

    q, qr, qb = make(Hq)
    k, kr, kb = make(Hk) if Hk else (None, None, None)
    if positions == "none":
        pos, pr = None, start + np.arange(T)[None].repeat(B, 0)
    else:
        pr = {"far": rng.integers(-(1 << 20), 1 << 20, size=(B, T)), "edge": rng.choice([-(1 << 31), (1 << 31) - 1, 0, -1], size=(B, T)),
              "shared": rng.integers(0, 5000, size=(1, T)).repeat(B, 0)}[positions]
        pos = torch.from_numpy(pr.astype(np.int32)).cuda()
        if positions == "shared":
            pos = pos[:1].expand(B, T)
    table = ops.rope_table(**spec)
    fn = ops.rope_backward if backward else ops.rope
    qo, ko = fn(q, k, table, positions=pos, start=start, layout=layout, out=(q, k) if inplace else None)
    torch.cuda.synchronize()
    sign = -1.0 if backward else 1.0
    for y, r, H, buf, name in ((qo, qr, Hq, qb, "q"), (ko, kr, Hk, kb, "k")):
        if y is None:
            continue
        _check_rope(_np(y), r, pr, spec, layout, sign, dtype, what + (name,))
        v = q if name == "q" else k
        v.fill_(7.0)
        assert bool((buf == 7.0).all()), what  # nothing beside the heads was written


SPEC = dict(rot_dim=64)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("B,T,Hq,Hk,D,rot", [
    (1, 1, 1, 0, 2, 2), (2, 3, 4, 2, 64, 64), (3, 17, 5, 1, 80, 48), (1, 5, 2, 2, 96, 20), (2, 7, 3, 1, 33, 10),
    (1, 3, 2, 1, 1024, 1024), (1, 4, 1, 1, 1024, 2), (5, 1, 8, 2, 128, 64), (1, 1, 40, 8, 128, 128), (2, 130, 3, 3, 40, 8),
    (70, 1, 2, 1, 16, 16), (1, 2, 130, 33, 64, 32), (4, 33, 2, 1, 24, 24), (1, 9, 1, 0, 7, 6), (2, 5, 6, 2, 72, 64)])
def test_rope_shapes(dtype, layout, B, T, Hq, Hk, D, rot):
    _rope_case(dtype, layout, B, T, Hq, Hk, D, dict(rot_dim=rot), "none")
    _rope_case(dtype, layout, B, T, Hq, Hk, D, dict(rot_dim=rot), "far", backward=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("lay", ["bthd", "bhtd", "gaps"])
@pytest.mark.parametrize("lead,inplace", [(0, True), (1, False), (3, True)])
def test_rope_strides_and_alignment(dtype, layout, lay, lead, inplace):
    _rope_case(dtype, layout, 3, 21, 4, 2, 64, dict(rot_dim=64), "far", lay=lay, lead=lead, inplace=inplace)
    _rope_case(dtype, layout, 2, 5, 3, 1, 48, dict(rot_dim=24), "none", lay=lay, lead=lead, inplace=inplace, backward=True)


@pytest.mark.parametrize("spec", [
    dict(rot_dim=64, scaling="linear", factor=4.0), dict(rot_dim=64, scaling="ntk", factor=8.0),
    dict(rot_dim=64, scaling="by_parts", factor=8.0, original_length=4096.0), dict(rot_dim=48, base=1.0),
    dict(rot_dim=64, base=500000.0), dict(rot_dim=2, scaling="ntk", factor=3.0)])
@pytest.mark.parametrize("positions,start", [("none", 0), ("none", -5), ("none", 1 << 30), ("far", 0), ("edge", 0), ("shared", 0)])
def test_rope_scalings_and_positions(spec, positions, start):
    _rope_case("f32", "half", 2, 9, 2, 1, 64, spec, positions, start=start)
    _rope_case("f32", "interleaved", 2, 9, 2, 1, 64, spec, positions, start=start, backward=True)


def test_rope_of_a_packed_projection_and_of_nothing():
    import torch
    rng = np.random.Generator(np.random.PCG64(5))
    x, ref = _dev(rng.normal(size=(2, 50, 5 * 64)), "bf16")
    q, k = x[..., :192].unflatten(-1, (3, 64)), x[..., 192:256].unflatten(-1, (1, 64))
    table = ops.rope_table(64)
    ops.rope(q, k, table, out=(q, k))
    torch.cuda.synchronize()
    pos = np.arange(50)[None].repeat(2, 0)
    _check_rope(_np(q), ref[..., :192].reshape(2, 50, 3, 64), pos, SPEC, "half", 1.0, "bf16", "packed q")
    _check_rope(_np(k), ref[..., 192:256].reshape(2, 50, 1, 64), pos, SPEC, "half", 1.0, "bf16", "packed k")
    assert np.array_equal(_np(x)[..., 256:], ref[..., 256:])
    for B, T in ((0, 3), (3, 0)):
        e = torch.empty((B, T, 2, 64), device="cuda")
        qo, ko = ops.rope(e, e, table)
        assert qo.shape == e.shape and ko.shape == e.shape


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("D,rot", [(64, 64), (48, 20), (27, 6), (80, 34)])
def test_rope_mixed_places_and_layouts(dtype, layout, D, rot):
    """q written elsewhere in another order of dimensions while k stays in place,
    and the other way round; more key heads than query heads."""
    import torch
    rng = np.random.Generator(np.random.PCG64(D + rot))
    B, T, Hq, Hk = 3, 19, 2, 5
    spec, pos = dict(rot_dim=rot), np.arange(T)[None].repeat(B, 0) + 7
    table = ops.rope_table(rot)
    for q_in_place in (False, True):
        q, qr = _dev(rng.normal(size=(B, T, Hq, D)), dtype)
        k, kr = _dev(rng.normal(size=(B, T, Hk, D)), dtype)
        other = lambda x: torch.full((x.shape[0], x.shape[2], x.shape[1], D + 1), 7.0, dtype=x.dtype, device="cuda")
        buf = other(k if q_in_place else q)  # [B][H][T][D + 1]
        away = buf[..., :D].transpose(1, 2)
        out = (q, away) if q_in_place else (away, k)
        ops.rope(q, k, table, start=7, layout=layout, out=out)
        torch.cuda.synchronize()
        _check_rope(_np(out[0]), qr, pos, spec, layout, 1.0, dtype, (D, rot, q_in_place, "q"))
        _check_rope(_np(out[1]), kr, pos, spec, layout, 1.0, dtype, (D, rot, q_in_place, "k"))
        assert bool((buf[..., D] == 7.0).all())


def test_rope_positions_of_long_rows():
    """Rows of positions 200000 apart, and a single row whose stride says nothing."""
    import torch
    T = 200000
    table = ops.rope_table(2)
    x = torch.ones((2, T, 1, 2), device="cuda")
    pos = torch.arange(2 * T, dtype=torch.int32, device="cuda").view(2, T)
    at = [0, 1, 131071, 131072, T - 1]
    y, _ = ops.rope(x, None, table, positions=pos)
    got = _np(y[:, at])
    _check_rope(got, np.ones_like(got), _np(pos[:, at]), dict(rot_dim=2), "half", 1.0, "f32", "long rows")
    y1, _ = ops.rope(x[:1], None, table, positions=pos.view(-1)[:T].as_strided((1, T), (1 << 40, 1)))
    assert torch.equal(y1, y[:1])


def test_rope_broadcast_input_and_infinities():
    import torch
    x, ref = _dev(np.random.Generator(np.random.PCG64(6)).normal(size=(1, 1, 1, 64)), "f32")
    q = x.expand(3, 11, 2, 64)  # stride 0 in every dimension
    qo, _ = ops.rope(q, None, ops.rope_table(64))
    pos = np.arange(11)[None].repeat(3, 0)
    _check_rope(_np(qo), np.broadcast_to(ref, (3, 11, 2, 64)), pos, SPEC, "half", 1.0, "f32", "broadcast")
    # a NaN stays in its own pair
    y = torch.zeros((1, 4, 1, 64), device="cuda")
    y[0, 2, 0, 5] = float("nan")
    yo, _ = ops.rope(y, None, ops.rope_table(64))
    bad = torch.isnan(yo).nonzero().cpu().tolist()
    assert bad == [[0, 2, 0, 5], [0, 2, 0, 37]]


# ---------------------------------------------------------------------------
# layer norm
# ---------------------------------------------------------------------------
def _norm_bounds(x, w, b, mean, rstd, y, dtype, cols, eps):
    """Bounds of (y, mean, rstd): sums of cols terms in any order."""
    n = cols + 2  # additions, the division and its product
    dm = n * U * np.abs(x).mean(1)                                     # mean
    var = ((x - mean[:, None]) ** 2).mean(1)
    # the centred row is off by dm and one rounding; the mean's error adds dm^2 to the variance
    dv = (n + 2) * U * var + (dm + U * np.abs(mean)) ** 2 * 1.01
    dr = rstd * (0.5 * dv / (var + eps) + 3 * U)
    h = np.abs(x - mean[:, None]) * rstd[:, None]
    dh = (dm[:, None] + U * np.abs(x - mean[:, None])) * rstd[:, None] + h * (dr / rstd)[:, None] + U * h
    ww = 1.0 if w is None else np.abs(w)
    return dh * ww * 1.01 + 2 * U * (h * ww + (0.0 if b is None else np.abs(b))) + HALF[dtype] * np.abs(y), dm, dr


def _norm_case(dtype, R, C, weight=True, bias=True, lead=0, gap=0, inplace=False, shift=0.3, scale=1.0, eps=1e-5, x=None):
    import torch
    what = (dtype, R, C, weight, bias, lead, gap, inplace, shift, scale)
    print("[norm]", what, flush=True)
    rng = np.random.Generator(np.random.PCG64(R * 7 + C))
    xa, xr = _dev(rng.normal(size=(R, C)) * scale + shift if x is None else x, dtype)
    w, wr = _dev(1 + 0.3 * rng.normal(size=C), "f32") if weight else (None, None)
    b, br = _dev(rng.normal(size=C), "f32") if bias else (None, None)
    ld = C + gap
    xv, xb = _inside(xa, lead, ld)
    out = None
    if inplace:
        out = (xv, torch.empty(R, device="cuda"), torch.empty(R, device="cuda"))
    elif lead or gap:
        yv, yb = _inside(torch.zeros_like(xa), lead, ld)
        out = (yv, torch.empty(R, device="cuda"), torch.empty(R, device="cuda"))
    y, m, r = ops.layer_norm(xv, w, b, eps=eps, out=out)
    torch.cuda.synchronize()
    want, wm, wr_ = oo.layer_norm(xr, wr, br, eps)
    by, bm, br2 = _norm_bounds(xr, wr, br, wm, wr_, want, dtype, C, eps)
    for name, got, ref, bound in (("y", _np(y), want, by), ("mean", _np(m), wm, bm), ("rstd", _np(r), wr_, br2)):
        e = np.abs(got - ref) - bound
        assert not e.size or e.max() <= TINY, (what, name, float(e.max()))
    assert _rest_untouched(xb, lead, R, C, ld), what
    if out is not None and not inplace:
        assert _rest_untouched(yb, lead, R, C, ld), what


COLS = [1, 2, 3, 4, 5, 7, 8, 9, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 401, 511, 512, 513, 1000, 1023, 1024, 1025, 1677, 2047, 2048, 2049,
        4096, 4097, 8191, 8192, 8193, 12345, 16383, 16384]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("C", COLS)
def test_layer_norm_widths(dtype, C):
    _norm_case(dtype, 5, C)
    _norm_case(dtype, 1, C, bias=False, gap=3)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("R,C", [(0, 64), (1, 1), (2, 512), (3, 100), (63, 64), (257, 512), (1000, 130), (4099, 40), (2051, 520)])
def test_layer_norm_rows(dtype, R, C):
    _norm_case(dtype, R, C, weight=R % 2 == 0, bias=R % 3 == 0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("C", [40, 100, 512, 1001, 2050, 4100, 9000])
@pytest.mark.parametrize("lead,gap,inplace", [(1, 0, False), (0, 5, True), (3, 1, True), (5, 8, False)])
def test_layer_norm_pitches_and_alignment(dtype, C, lead, gap, inplace):
    _norm_case(dtype, 9, C, lead=lead, gap=gap, inplace=inplace)


def test_layer_norm_far_from_zero_and_constant_rows():
    # mean 1000 deviations away: sums of squares would cancel
    _norm_case("f32", 33, 700, shift=1000.0)
    _norm_case("f32", 6, 4000, shift=-1e4, scale=10.0)
    # constant rows: the variance is 0 (up to the mean's rounding), eps decides
    import torch
    x = torch.full((3, 513), 3.0, device="cuda")
    y, m, r = ops.layer_norm(x, None, None, eps=1e-5)
    # 513 times 3 is a sum of whole numbers below 2^24: exact, so the row is centred exactly
    assert bool((m == 3.0).all()) and bool((y == 0).all())
    assert np.abs(_np(r) * np.sqrt(float(np.float32(1e-5))) - 1).max() <= 4 * U
    # eps 0 and a constant row: 1 / 0, the centred zeros give NaN as the formula does
    y, m, r = ops.layer_norm(x, None, None, eps=0.0)
    assert bool(torch.isinf(r).all()) and bool(torch.isnan(y).all())


def test_layer_norm_keeps_a_bad_row_to_itself():
    import torch
    x = torch.randn((67, 300), device="cuda")
    clean, _, _ = ops.layer_norm(x)
    x[13, 7] = float("nan")
    x[40, 299] = float("inf")
    y, m, r = ops.layer_norm(x)
    bad = torch.isnan(y).any(1).nonzero().flatten().tolist()
    assert bad == [13, 40]
    ok = [i for i in range(67) if i not in bad]
    assert torch.equal(y[ok], clean[ok])


def test_layer_norm_without_statistics():
    import torch
    x = torch.randn((9, 200), device="cuda").bfloat16()
    y, m, r = ops.layer_norm(x)
    y2, m2, r2 = ops.layer_norm(x, out=(torch.empty_like(x), None, None))
    assert m2 is None and r2 is None and torch.equal(y, y2)


def _norm_bwd_case(dtype, R, C, weight=True, res=False, lead=0, gap=0, alias=None, need=(True, True, True), shift=0.3):
    import torch
    what = (dtype, R, C, weight, res, lead, gap, alias, need)
    print("[norm backward]", what, flush=True)
    rng = np.random.Generator(np.random.PCG64(R * 11 + C))
    xa, xr = _dev(rng.normal(size=(R, C)) * 2 + shift, dtype)
    da, dr = _dev(rng.normal(size=(R, C)), dtype)
    ra, rr = _dev(rng.normal(size=(R, C)), dtype) if res else (None, None)
    w, wr = _dev(1 + 0.3 * rng.normal(size=C), "f32") if weight else (None, None)
    _, m, r = oo.layer_norm(xr)
    mean, mr = _dev(m, "f32")
    rstd, sr = _dev(r, "f32")
    ld = C + gap
    xv, xb = _inside(xa, lead, ld)
    dv, db_ = _inside(da, lead, ld)
    rv, rb = _inside(ra, lead, ld) if res else (None, None)
    out = None
    if alias:
        dx = dv if alias == "dy" else rv
        out = (dx, None, None)
    elif lead or gap:
        ov, ob = _inside(torch.zeros_like(xa), lead, ld)
        out = (ov, None, None)
    got = ops.layer_norm_backward(dv, xv, w, mean, rstd, residual=rv, need_input=need[0], need_weight=need[1],
                                  need_bias=need[2], out=out)
    torch.cuda.synchronize()
    want = oo.layer_norm_backward(dr, xr, wr, mr, sr, rr)
    h = np.abs(xr - mr[:, None]) * sr[:, None]
    g = np.abs(dr if wr is None else dr * wr)
    n = C + 2
    # g: 1 rounding, h: 2, g h: 4, their means n more, then 4 roundings up to the product with r and 1 for the sum with res
    dmg, dmgh = (n + 1) * U * g.mean(1), (n + 4) * U * (g * h).mean(1)
    mgh = np.abs((np.where(True, dr if wr is None else dr * wr, 0) * ((xr - mr[:, None]) * sr[:, None])).mean(1)) if R else np.zeros(0)
    inner = g * 4 * U + (np.abs(g).mean(1) * 4 * U + dmg)[:, None] + h * (dmgh + 7 * U * mgh)[:, None]
    bx = sr[:, None] * inner * 1.01 + 2 * U * (np.abs(rr) if res else 0) + (HALF[dtype] + U) * np.abs(want[0])
    # column sums: h 2 roundings, the product 1, R additions in any order
    bw = (R + 4) * U * (np.abs(dr) * h).sum(0)
    bb = (R + 1) * U * np.abs(dr).sum(0)
    for name, y, ref, bound, wanted in zip(("dx", "dw", "db"), got, want, (bx, bw, bb), need):
        if not wanted:
            assert y is None
            continue
        e = np.abs(_np(y) - ref) - bound
        assert not e.size or e.max() <= TINY, (what, name, float(e.max()))
    for v, buf, mine in ((xv, xb, False), (dv, db_, alias == "dy"), (rv, rb, alias == "res")):
        if buf is not None:
            assert _rest_untouched(buf, lead, R, C, ld), what
    if out is not None and not alias:
        assert _rest_untouched(ob, lead, R, C, ld), what
    assert np.array_equal(_np(xv), xr)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("C", COLS)
def test_layer_norm_backward_widths(dtype, C):
    _norm_bwd_case(dtype, 5, C)
    _norm_bwd_case(dtype, 1, C, weight=False, res=True, gap=3)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("R,C", [(0, 64), (1, 1), (2, 512), (3, 100), (63, 64), (257, 512), (1000, 130), (4099, 40), (2051, 520),
                                 (1500, 1100), (700, 4096), (5000, 16), (70001, 26), (9000, 6), (33000, 31)])
def test_layer_norm_backward_rows(dtype, R, C):
    _norm_bwd_case(dtype, R, C, weight=R % 2 == 0, res=R % 3 == 0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("C", [40, 100, 512, 1001, 2050, 4100, 9000])
@pytest.mark.parametrize("lead,gap,alias", [(1, 0, None), (0, 5, "dy"), (3, 1, "res"), (5, 8, None)])
def test_layer_norm_backward_pitches_and_aliases(dtype, C, lead, gap, alias):
    _norm_bwd_case(dtype, 9, C, lead=lead, gap=gap, alias=alias, res=True)
    _norm_bwd_case(dtype, 130, C, lead=lead, gap=gap, alias=None if alias == "res" else alias)


@pytest.mark.parametrize("R", [32, 33, 64, 65, 768, 769])
@pytest.mark.parametrize("dtype,C", [("bf16", 5), ("bf16", 512), ("f32", 515), ("bf16", 1030), ("f32", 3), ("bf16", 5000)])
def test_layer_norm_backward_around_one_launch(dtype, R, C):
    """Row counts on both sides of those that one launch serves, also with dx over dy."""
    _norm_bwd_case(dtype, R, C, gap=1)
    _norm_bwd_case(dtype, R, C, alias="dy")


@pytest.mark.parametrize("R", [2, 770, 1029])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("C", [8193, 12345, 16384])
def test_layer_norm_backward_of_the_widest_rows(dtype, C, R):
    """Sums of columns in one workgroup's rounds of rows, in uneven numbers."""
    _norm_bwd_case(dtype, R, C, res=R % 2 == 0, gap=C % 2)
    _norm_bwd_case(dtype, R, C, weight=False, need=(R % 2 == 0, True, R % 2 == 1))


@pytest.mark.parametrize("need", [(True, False, False), (False, True, False), (False, False, True), (True, True, False),
                                  (False, True, True), (True, False, True), (False, False, False)])
@pytest.mark.parametrize("R", [0, 7, 600])
def test_layer_norm_backward_parts(need, R):
    _norm_bwd_case("f32", R, 300, need=need)
    _norm_bwd_case("bf16", R, 2100, need=need)


@pytest.mark.parametrize("R,C", [(5, 333), (3000, 512), (700, 4096)])
def test_layer_norm_backward_is_deterministic(R, C):
    import torch
    x, dy = torch.randn((R, C), device="cuda").bfloat16(), torch.randn((R, C), device="cuda").bfloat16()
    w = torch.randn(C, device="cuda")
    _, m, r = ops.layer_norm(x, w)
    first = ops.layer_norm_backward(dy, x, w, m, r)
    scratch = ops.layer_norm_backward_scratch(x)
    for _ in range(3):
        scratch.fill_(255)  # NaN in every word: nothing of it may be read
        for a, b in zip(first, ops.layer_norm_backward(dy, x, w, m, r, scratch=scratch)):
            assert torch.equal(a, b)


# ---------------------------------------------------------------------------
# dropout
# ---------------------------------------------------------------------------
def _drop_case(dtype, R, C, p, seed, offset, res=False, lead=0, gap=0, alias=None, backward=False, step=None):
    import torch
    what = (dtype, R, C, p, seed, offset, res, lead, gap, alias, backward, step)
    print("[dropout]", what, flush=True)
    rng = np.random.Generator(np.random.PCG64(R * 13 + C))
    xa, xr = _dev(rng.normal(size=(R, C)) + 2.0, dtype)
    ra, rr = _dev(rng.normal(size=(R, C)), dtype) if res else (None, None)
    ld = C + gap
    xv, xb = _inside(xa, lead, ld)
    rv, rb = _inside(ra, lead, ld) if res else (None, None)
    ov, ob = (xv, xb) if alias == "x" else (rv, rb) if alias == "res" else _inside(torch.zeros_like(xa), lead, ld)
    st = None if step is None else torch.tensor([step], dtype=torch.int64, device="cuda")
    if backward:
        y = ops.dropout_backward(xv, p, seed, offset, step=st, out=ov)
    else:
        y = ops.dropout(xv, p, seed, offset, residual=rv, step=st, out=ov)
    torch.cuda.synchronize()
    want = oo.dropout(xr, p, seed, (offset + (step or 0)) % (1 << 64), rr)
    _, scale = oo.dropout_kept(1, 1, p, 0, 0)
    # the scale, its product and the sum: one rounding each
    bound = 3 * U * np.abs(xr) * scale + U * np.abs(want) + HALF[dtype] * np.abs(want)
    e = np.abs(_np(y) - want) - bound
    assert not e.size or e.max() <= TINY, (what, float(e.max()))
    for buf in (xb, rb, ob):
        if buf is not None:
            assert _rest_untouched(buf, lead, R, C, ld), what


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("R,C", [(0, 8), (3, 0), (1, 1), (1, 7), (1, 8), (1, 9), (5, 15), (7, 16), (3, 17), (64, 401), (33, 512), (300, 65),
                                 (1000, 8), (1001, 3), (2, 100003), (70001, 5), (9, 4096)])
def test_dropout_shapes(dtype, R, C):
    _drop_case(dtype, R, C, 0.3, 1234567890123456789, 42)
    _drop_case(dtype, R, C, 0.1, 3, 1 << 40, res=True)
    _drop_case(dtype, R, C, 0.5, 0, 0, backward=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("C", [24, 77, 512, 2051])
@pytest.mark.parametrize("lead,gap,alias,res", [(1, 0, None, True), (0, 5, "x", True), (3, 1, "res", True), (5, 8, None, False),
                                                (0, 0, "x", False), (8, 16, "res", True)])
def test_dropout_pitches_and_aliases(dtype, C, lead, gap, alias, res):
    _drop_case(dtype, 19, C, 0.4, 99, 7, res=res, lead=lead, gap=gap, alias=alias)


@pytest.mark.parametrize("p", [0.0, 2.0 ** -18, 2.0 ** -17, 2.0 ** -16, 0.25, 0.9999, 1 - 2.0 ** -16, 1 - 2.0 ** -18, 1.0])
def test_dropout_probabilities(p):
    _drop_case("f32", 40, 300, p, 11, 5, res=True)
    _drop_case("bf16", 40, 300, p, 11, 5)


@pytest.mark.parametrize("seed,offset,step", [(0, 0, 0), ((1 << 64) - 1, (1 << 64) - 1, 3), (5, 1 << 32, 1 << 33), (1 << 32, (1 << 32) - 1, 1),
                                              (7, 9, -1)])
def test_dropout_counters(seed, offset, step):
    if step < 0:
        step += 1 << 64
        import torch
        x = torch.ones((3, 50), device="cuda")
        got = ops.dropout(x, 0.5, seed, offset, step=torch.tensor([-1], dtype=torch.int64, device="cuda"))
        assert np.array_equal(_np(got) > 0, oo.dropout_kept(3, 50, 0.5, seed, (offset + step) % (1 << 64))[0])
        return
    _drop_case("f32", 6, 100, 0.5, seed, offset, step=step)


def _loose(rng, R, C, dtype, values=None):
    """A [R][C] tensor at an address and a pitch of its own: (view, buffer, lead, pitch, float64 values)."""
    import torch
    lead, ld = int(rng.integers(0, 9)), C + int(rng.integers(0, 12))
    t, ref = _dev(rng.normal(size=(R, C)) if values is None else values, dtype)
    v, buf = _inside(t, lead, ld)
    return v, buf, lead, ld, ref


@pytest.mark.parametrize("seed", range(24))
def test_every_operand_at_a_place_of_its_own(seed):
    import torch
    rng = np.random.Generator(np.random.PCG64(1000 + seed))
    dtype = ["bf16", "f32"][seed % 2]
    R, C = int(rng.integers(1, 200)), int(np.exp(rng.uniform(0, np.log(5000))))
    print("[places]", seed, dtype, R, C, flush=True)
    bufs = []

    def loose(values=None):
        v, buf, lead, ld, ref = _loose(rng, R, C, dtype, values)
        bufs.append((buf, lead, ld))
        return v, ref

    x, xr = loose(rng.normal(size=(R, C)) + 1)
    res, rr = loose()
    dy, dr = loose()
    y, _ = loose()
    dx, _ = loose()
    z, _ = loose()
    off = int(rng.integers(0, 4))
    vec = lambda: torch.from_numpy(rng.normal(size=C + off).astype(np.float32)).cuda()[off:]
    w, b = vec(), vec()
    _, m, r = ops.layer_norm(x, w, b, out=(y, torch.empty(R, device="cuda"), torch.empty(R, device="cuda")))
    got = ops.layer_norm_backward(dy, x, w, m, r, residual=res, out=(dx, vec(), vec()))
    ops.dropout(x, 0.3, seed, 5, residual=res, out=z)
    torch.cuda.synchronize()
    want, wm, wr = oo.layer_norm(xr, _np(w), _np(b))
    by = _norm_bounds(xr, _np(w), _np(b), wm, wr, want, dtype, C, 1e-5)[0]
    assert (np.abs(_np(y) - want) - by).max() <= TINY
    d64 = oo.layer_norm_backward(dr, xr, _np(w), _np(m), _np(r), rr)
    h = np.abs(xr - _np(m)[:, None]) * _np(r)[:, None]
    g = np.abs(dr * _np(w))
    n = C + 2
    # as in _norm_bwd_case, with |mean(g h)| bounded by the mean of |g h|
    inner = g * 4 * U + (g.mean(1) * (n + 5) * U)[:, None] + h * ((g * h).mean(1) * (n + 11) * U)[:, None]
    bx = _np(r)[:, None] * inner * 1.01 + 2 * U * np.abs(rr) + (HALF[dtype] + U) * np.abs(d64[0])
    assert (np.abs(_np(dx) - d64[0]) - bx).max() <= TINY
    assert (np.abs(_np(got[1]) - d64[1]) - (R + 4) * U * (np.abs(dr) * h).sum(0)).max() <= TINY
    assert (np.abs(_np(got[2]) - d64[2]) - (R + 1) * U * np.abs(dr).sum(0)).max() <= TINY
    drop = oo.dropout(xr, 0.3, seed, 5, rr)
    assert (np.abs(_np(z) - drop) - 3 * U * np.abs(xr) * 1.5 - (U + HALF[dtype]) * np.abs(drop)).max() <= TINY
    for buf, lead, ld in bufs:
        assert _rest_untouched(buf, lead, R, C, ld)


def test_dropped_elements_contribute_nothing():
    import torch
    kept, _ = oo.dropout_kept(20, 333, 0.5, 8, 1)
    for bad in (float("nan"), float("inf"), -float("inf")):
        x = torch.where(torch.from_numpy(kept).cuda(), 1.0, bad)
        y = ops.dropout(x, 0.5, 8, 1)
        assert np.array_equal(_np(y), np.where(kept, 2.0, 0.0))
        y = ops.dropout(torch.full((4, 9), bad, device="cuda"), 1.0, 8, 1, residual=torch.ones((4, 9), device="cuda"))
        assert bool((y == 1).all())


# ---------------------------------------------------------------------------
# positions in memory, streams, graphs
# ---------------------------------------------------------------------------
def test_rows_beyond_32_bit_offsets():
    """The last of 1030 rows, 2^22 elements apart: element offsets pass 2^32."""
    import torch
    R, ld, C = 1030, 1 << 22, 96
    assert (R - 1) * ld > 1 << 32
    buf = torch.zeros(R * ld, dtype=torch.bfloat16, device="cuda")
    x = buf.view(R, ld)[:, :C]
    x.copy_(torch.randn((R, C), device="cuda"))
    y = buf.view(R, ld)[:, 1024:1024 + C]
    xr = _np(x)
    print("[far rows] norm", flush=True)
    ops.layer_norm(x, out=(y, None, None))
    want, m, r = oo.layer_norm(xr)
    assert (np.abs(_np(y) - want) - _norm_bounds(xr, None, None, m, r, want, "bf16", C, 1e-5)[0]).max() <= 0
    print("[far rows] dropout", flush=True)
    ops.dropout(x, 0.5, 4, out=y)
    assert np.array_equal(_np(y), oo.dropout(xr, 0.5, 4))  # times 2: exact
    print("[far rows] norm backward", flush=True)
    mean, rstd = torch.from_numpy(m).cuda().float(), torch.from_numpy(r).cuda().float()
    dx, dw, _ = ops.layer_norm_backward(x, x, None, mean, rstd, out=(y, None, None))
    d64, w64, _ = oo.layer_norm_backward(xr, xr, None, _np(mean), _np(rstd))
    assert np.abs(_np(dw) - w64).max() <= (R + 4) * U * (xr * xr * _np(rstd)[:, None] + np.abs(xr * (m * r)[:, None])).sum(0).max()
    print("[far rows] rope", flush=True)
    q = buf.view(1, R, ld)[:, :, :64].unflatten(-1, (1, 64))
    qr = _np(q)
    qo, _ = ops.rope(q, None, ops.rope_table(64), out=(q, None))
    _check_rope(_np(qo), qr, np.arange(R)[None], SPEC, "half", 1.0, "bf16", "far rows")


def test_dropout_of_more_than_2_to_the_32_elements():
    import torch
    R, C = 8200, 1 << 19
    x = torch.ones((R, C), dtype=torch.bfloat16, device="cuda")
    ops.dropout(x, 0.5, 21, 6, out=x)
    for r in (0, 4095, 4096, R - 1):
        words = oo.dropout_kept(1, C, 0.5, 21, 6, row0=r)[0]
        assert np.array_equal(x[r].float().cpu().numpy() > 0, words[0]), r


def test_the_longest_sequence_and_row():
    """2^31 - 1 positions in one sequence, 2^31 - 1 columns in one row."""
    import torch
    n = (1 << 31) - 1
    print("[longest] rope", flush=True)
    x = torch.ones((1, n, 1, 2), dtype=torch.bfloat16, device="cuda")
    at = [0, 1, 12345, 1 << 30, n - 2, n - 1]
    ops.rope(x, None, ops.rope_table(2), out=(x, None))
    got = _np(x[:, at])
    _check_rope(got, np.ones_like(got), np.array([at]), dict(rot_dim=2), "half", 1.0, "bf16", "longest")
    del x
    print("[longest] dropout", flush=True)
    x = torch.ones((1, n), dtype=torch.bfloat16, device="cuda")
    ops.dropout(x, 0.5, 3, out=x)
    group = n // 8  # of the last columns
    words = oo.philox(np.array([[group, 0, 0, 0]], np.uint64), (3, 0))[0]
    halves = np.stack([words & 0xFFFF, words >> 16], -1).reshape(-1)
    assert np.array_equal(_np(x[0, 8 * group:]) > 0, (halves >= 32768)[:n - 8 * group])


def test_layer_norm_of_more_rows_than_one_grid_row_takes():
    """2^26 + 5 rows, a wave each: 2^32 threads and more."""
    import torch
    R, C = (1 << 26) + 5, 129
    x = torch.zeros((R, C), dtype=torch.bfloat16, device="cuda")
    at = [0, 1, 4 << 22, (1 << 26) - 1, 1 << 26, R - 1]
    x[at] = torch.randn((len(at), C), device="cuda").bfloat16()
    xr = _np(x[at])
    print("[many rows]", R, C, flush=True)
    ops.layer_norm(x, out=(x, None, None))
    want, m, r = oo.layer_norm(xr)
    assert (np.abs(_np(x[at]) - want) - _norm_bounds(xr, None, None, m, r, want, "bf16", C, 1e-5)[0]).max() <= 0
    assert int(torch.count_nonzero(x[2:1000])) == 0 and int(torch.count_nonzero(x[-1000:-5])) <= C


def test_two_streams_at_once():
    import torch
    x = torch.randn((4000, 512), device="cuda").bfloat16()
    dy = torch.randn((4000, 512), device="cuda").bfloat16()
    w = torch.randn(512, device="cuda")
    q = torch.randn((4, 1000, 8, 64), device="cuda").bfloat16()
    table = ops.rope_table(64)
    y0, m0, r0 = ops.layer_norm(x, w)
    g0 = ops.layer_norm_backward(dy, x, w, m0, r0)
    q0, _ = ops.rope(q, None, table)
    d0 = ops.dropout(x, 0.1, 5)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        for s in streams:
            with torch.cuda.stream(s):
                y, m, r = ops.layer_norm(x, w)
                got.append((y, *ops.layer_norm_backward(dy, x, w, m, r), ops.rope(q, None, table)[0], ops.dropout(x, 0.1, 5)))
    # a stream given by name, while another is current
    s = streams[0]
    out = torch.empty_like(x)
    torch.cuda.synchronize()
    ops.dropout(x, 0.1, 5, out=out, stream=s)
    s.synchronize()
    assert torch.equal(out, d0)
    torch.cuda.synchronize()
    for one in got:
        for a, b in zip(one, (y0, *g0, q0, d0)):
            assert torch.equal(a, b)


def test_two_host_threads_at_once():
    """Calls of two threads, each on a stream of its own, share nothing."""
    import threading

    import torch
    x = [torch.randn((700, 1000), device="cuda").bfloat16() for _ in range(2)]
    q = torch.randn((4, 100, 4, 64), device="cuda")
    table = ops.rope_table(64)
    torch.cuda.synchronize()

    def work(i, n):
        out = []
        for j in range(n):
            y, m, r = ops.layer_norm(x[i])
            out = [y, *ops.layer_norm_backward(x[1 - i], x[i], None, m, r), ops.rope(q, None, table, start=i)[0],
                   ops.dropout(x[i], 0.3, i)]
        return out

    want = [work(i, 1) for i in range(2)]
    torch.cuda.synchronize()
    got = [None, None]

    def run(i):
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            got[i] = work(i, 50)
        s.synchronize()

    ts = [threading.Thread(target=run, args=(i,)) for i in range(2)]
    for t in ts:
        t.start()
    for t in ts:
        t.join()
    for a, b in zip(want, got):
        assert b is not None and all(torch.equal(u, v) for u, v in zip(a, b))


def test_named_stream_owns_what_is_allocated_for_it():
    """With a stream given by name the outputs and the scratch come from that
    stream's memory: the current stream's next allocations do not touch them."""
    import torch
    x, dy = torch.randn((3000, 512), device="cuda"), torch.randn((3000, 512), device="cuda")
    w = torch.ones(512, device="cuda")
    y0, m, r = ops.layer_norm(x, w)
    want = ops.layer_norm_backward(dy, x, w, m, r)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(20):
        got = ops.layer_norm_backward(dy, x, w, m, r, stream=s)
        junk = [torch.full((1 << 20,), float("nan"), device="cuda") for _ in range(4)]  # would reuse freed scratch
        del junk
    s.synchronize()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_captured_and_replayed():
    """Forward and backward of the three in one graph: every replay equals the
    eager calls, with a new dropout mask whenever the counter moved."""
    import torch
    R, C = 1000, 512
    x, dy = torch.randn((R, C), device="cuda").bfloat16(), torch.randn((R, C), device="cuda").bfloat16()
    w, b = torch.randn(C, device="cuda"), torch.randn(C, device="cuda")
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    table = ops.rope_table(64)

    def block():
        d = ops.dropout(x, 0.2, 17, 100, residual=x, step=step)
        y, m, r = ops.layer_norm(d, w, b)
        q, k = ops.rope(y.view(10, 100, 8, 64), y.view(10, 100, 8, 64), table)
        dq, dk = ops.rope_backward(q, k, table)
        dx, dw, db = ops.layer_norm_backward(dy, d, w, m, r, residual=dq.view(R, C))
        return d, y, q, k, dk, dx, dw, db, ops.dropout_backward(dx, 0.2, 17, 100, step=step)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        block()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        captured = block()
    masks = []
    for i in range(4):
        step.fill_(i // 2)
        x.copy_(torch.randn((R, C), device="cuda"))
        g.replay()
        torch.cuda.synchronize()
        for a, e in zip(captured, block()):
            assert torch.equal(a, e), i
        masks.append((ops.dropout(torch.ones_like(x), 0.2, 17, 100, step=step) > 0).clone())
    assert torch.equal(masks[0], masks[1]) and torch.equal(masks[2], masks[3]) and not torch.equal(masks[1], masks[2])


def test_a_block_forward_and_backward():
    """The three together as a pre-norm block uses them, in fp32 against torch
    autograd in float64 (masks from the oracle): x1 = x + dropout(attention of
    rotated queries and keys of norm(x)), y = norm(x1)."""
    import torch
    B, T, H, D, p = 2, 37, 3, 32, 0.25
    C, N = H * D, B * T
    g = torch.Generator(device="cuda").manual_seed(3)
    mk = lambda *s: torch.randn(s, generator=g, device="cuda")
    x, dy, w1, b1, w2, b2 = mk(N, C), mk(N, C), mk(C), mk(C), mk(C), mk(C)
    Wq, Wo = mk(3 * C, C) / C ** 0.5, mk(C, C) / C ** 0.5
    freq, _ = oo.rope_frequencies(D)
    hide = torch.ones((T, T), dtype=torch.bool, device="cuda").triu(1)

    def attend(q, k, v):  # [B][T][H][D] in, [N][C] out
        q, k, v = (t.transpose(1, 2).contiguous() for t in (q, k, v))
        s = torch.matmul(q, k.transpose(2, 3).contiguous()) / D ** 0.5
        return torch.matmul(torch.softmax(s.masked_fill(hide, float("-inf")), -1), v).transpose(1, 2).reshape(N, C)

    # float64
    leaves = [t.double().requires_grad_() for t in (x, w1, b1, w2, b2)]
    X, W1, B1, W2, B2 = leaves
    kept, scale = oo.dropout_kept(N, C, p, 9, 4)
    mask = torch.from_numpy(kept * scale).cuda()
    th = torch.arange(T, dtype=torch.float64, device="cuda")[:, None] * torch.from_numpy(freq).cuda()
    cs, sn = torch.cos(th)[:, None], torch.sin(th)[:, None]
    turn = lambda t: torch.cat([t[..., :D // 2] * cs - t[..., D // 2:] * sn, t[..., D // 2:] * cs + t[..., :D // 2] * sn], -1)
    qkv = (torch.nn.functional.layer_norm(X, (C,), W1, B1) @ Wq.double().t()).view(B, T, 3, H, D)
    X1 = X + mask * (attend(turn(qkv[:, :, 0]), turn(qkv[:, :, 1]), qkv[:, :, 2]) @ Wo.double().t())
    Y = torch.nn.functional.layer_norm(X1, (C,), W2, B2)
    want = torch.autograd.grad((Y * dy.double()).sum(), leaves)

    # the operators in fp32, the products and the attention by torch
    table = ops.rope_table(D)
    n1, m1, r1 = ops.layer_norm(x, w1, b1)
    qkv = (n1 @ Wq.t()).view(B, T, 3, H, D)
    q, k = ops.rope(qkv[:, :, 0], qkv[:, :, 1], table)
    v = qkv[:, :, 2].contiguous()
    q.requires_grad_(), k.requires_grad_(), v.requires_grad_()
    o = attend(q, k, v)
    x1 = ops.dropout(o.detach() @ Wo.t(), p, 9, 4, residual=x)
    y, m2, r2 = ops.layer_norm(x1, w2, b2)
    dx1, dw2, db2 = ops.layer_norm_backward(dy, x1, w2, m2, r2)
    do = ops.dropout_backward(dx1, p, 9, 4) @ Wo
    dq, dk, dv = torch.autograd.grad(o, (q, k, v), do)
    dq, dk = ops.rope_backward(dq.contiguous(), dk.contiguous(), table)
    dqkv = torch.stack([dq, dk, dv], 2).reshape(N, 3 * C)
    dx, dw1, db1 = ops.layer_norm_backward(dqkv @ Wq, x, w1, m1, r1, residual=dx1)
    # about a dozen fp32 stages of sums over at most 3 C = 288 terms, each within 300 u of its norm
    for name, a, e in zip(("y", "x", "w1", "b1", "w2", "b2"), (y, dx, dw1, db1, dw2, db2), (Y.detach(), *want)):
        rel = float((a.double() - e).norm() / e.norm())
        assert rel <= 12 * 300 * U, (name, rel)
