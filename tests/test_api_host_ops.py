"""Host-only checks of the operators' C ABI (include/erase_ops.h): the library
exports every declared entry point, computes the rotary frequencies, and
refuses bad calls before any HIP call (no GPU needed)."""
import ctypes
import os
import re

import numpy as np
import pytest

from oracle import ops_oracle as oo
from paper_2608_18469_amd import erase, erase_ops as ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P, Q, R, S = 0x100000, 0x200000, 0x300000, 0x400000  # addresses no refused call may reach
INVALID, SHAPE, WORKSPACE = erase.ERR_INVALID_ARG, erase.ERR_SHAPE, erase.ERR_WORKSPACE


def test_library_exports_every_declared_operator():
    with open(os.path.join(ROOT, "include", "erase_ops.h")) as f:
        text = re.sub(r"/\*.*?\*/", "", f.read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(erase_[a-z_]+)\s*\(", text)))
    L = ops.lib()
    assert len(names) >= 10 and set(names) == set(ops.SIGNATURES)
    for n in names:
        assert hasattr(L, n), n


@pytest.mark.parametrize("kw", [
    dict(rot_dim=64), dict(rot_dim=2), dict(rot_dim=1024, base=500000.0), dict(rot_dim=48, scaling="linear", factor=4.0),
    dict(rot_dim=128, scaling="ntk", factor=8.0), dict(rot_dim=2, scaling="ntk", factor=8.0),
    dict(rot_dim=64, scaling="by_parts", factor=8.0, original_length=4096.0),
    dict(rot_dim=96, scaling="by_parts", factor=32.0, original_length=2048.0, fast=16.0, slow=0.0),
    dict(rot_dim=64, base=1.0), dict(rot_dim=64, scaling="by_parts", factor=1.0, original_length=1.0)])
def test_frequencies(kw):
    f, a = ops.rope_frequencies(**kw)
    want, amp = oo.rope_frequencies(**kw)
    # a few roundings of pow, log and products in double
    assert np.allclose(f, want, rtol=1e-13, atol=0) and abs(a - amp) <= 1e-15 * amp
    n = ctypes.c_size_t(0)
    spec = ops._rope_spec(*[kw.get(k, d) for k, d in (("rot_dim", 0), ("base", 10000.0), ("scaling", "none"), ("factor", 1.0),
                                                      ("original_length", 0.0), ("fast", 32.0), ("slow", 1.0))])
    assert ops.lib().erase_rope_table_bytes(ctypes.byref(spec), ctypes.byref(n)) == 0
    assert n.value == 8 * (kw["rot_dim"] // 2 + 1)


@pytest.mark.parametrize("kw,code", [
    (dict(rot_dim=0), SHAPE), (dict(rot_dim=3), SHAPE), (dict(rot_dim=1026), SHAPE), (dict(rot_dim=-2), SHAPE),
    (dict(scaling=4), INVALID), (dict(scaling=-1), INVALID), (dict(base=0.5), INVALID), (dict(base=float("nan")), INVALID),
    (dict(base=float("inf")), INVALID), (dict(scaling=1, factor=0.5), INVALID), (dict(scaling=1, factor=float("nan")), INVALID),
    (dict(scaling=2, factor=float("inf")), INVALID), (dict(scaling=3, factor=2.0), INVALID),
    (dict(scaling=3, factor=2.0, original_length=10.0, fast=1.0, slow=1.0), INVALID),
    (dict(scaling=3, factor=2.0, original_length=10.0, slow=-1.0), INVALID),
    (dict(scaling=3, factor=2.0, original_length=float("inf")), INVALID)])
def test_bad_specs(kw, code):
    d = dict(rot_dim=64, scaling=0, base=10000.0, factor=1.0, original_length=0.0, fast=32.0, slow=1.0)
    d.update(kw)
    spec = ops.RopeSpec(*d.values())
    L = ops.lib()
    out, amp, n = (ctypes.c_double * 1024)(), ctypes.c_double(0), ctypes.c_size_t(0)
    assert L.erase_rope_frequencies(ctypes.byref(spec), out, ctypes.byref(amp)) == code
    assert L.erase_rope_table_bytes(ctypes.byref(spec), ctypes.byref(n)) == code
    assert L.erase_rope_table(ctypes.byref(spec), P, None) == code


def test_table_pointers():
    spec = ops.RopeSpec(64, 0, 10000.0, 1.0, 0.0, 32.0, 1.0)
    L = ops.lib()
    assert L.erase_rope_table(ctypes.byref(spec), None, None) == INVALID
    assert L.erase_rope_table(ctypes.byref(spec), P + 4, None) == INVALID
    assert L.erase_rope_table(None, P, None) == INVALID


def _rope(fn="erase_rope", q=P, k=Q, qo=R, ko=S, pos=None, table=P, **kw):
    c = ops.RopeConfig(erase.BF16, 0, 2, 3, 4, 2, 64, 64, (768, 256, 64), (384, 128, 64), (768, 256, 64), (384, 128, 64), 3, 0)
    for name, v in kw.items():
        setattr(c, name, (ctypes.c_int64 * 3)(*v) if isinstance(v, tuple) else v)
    return getattr(ops.lib(), fn)(ctypes.byref(c), q, k, qo, ko, pos, table, None)


@pytest.mark.parametrize("fn", ["erase_rope", "erase_rope_backward"])
@pytest.mark.parametrize("kw,code", [
    (dict(dtype=2), INVALID), (dict(dtype=-1), INVALID), (dict(layout=2), INVALID), (dict(layout=-1), INVALID),
    (dict(batch=-1), SHAPE), (dict(seq=-1), SHAPE), (dict(batch=1 << 16, seq=1 << 15), SHAPE), (dict(q_heads=0), SHAPE),
    (dict(q_heads=4097), SHAPE), (dict(k_heads=-1), SHAPE), (dict(head_dim=1026), SHAPE), (dict(rot_dim=0), SHAPE),
    (dict(rot_dim=63), SHAPE), (dict(rot_dim=66), SHAPE), (dict(pos_stride=-1), SHAPE), (dict(pos_stride=1 << 48), SHAPE),
    (dict(start=1 << 41), INVALID),
    (dict(start=-(1 << 41)), INVALID), (dict(q_stride=(-768, 256, 64)), SHAPE), (dict(k_stride=(384, 128, -64)), SHAPE),
    (dict(q_stride=(1 << 62, 256, 64)), SHAPE),                  # beyond any memory
    (dict(qo_stride=(768, 256, 32)), SHAPE),                     # heads of the output overlap
    (dict(qo_stride=(0, 256, 64)), SHAPE),                       # batch rows of the output coincide
    (dict(ko_stride=(128, 128, 64)), SHAPE),
    (dict(ko_stride=(384, 127, 64)), SHAPE),
    (dict(q=None), INVALID), (dict(k=None), INVALID), (dict(qo=None), INVALID), (dict(ko=None), INVALID),
    (dict(table=None), INVALID), (dict(table=P + 4), INVALID), (dict(q=P + 1), INVALID), (dict(ko=S + 1), INVALID),
    (dict(dtype=0, k=Q + 2), INVALID), (dict(pos=P + 2), INVALID),
    (dict(q=R, q_stride=(1536, 512, 64)), INVALID)])             # in place with other strides
def test_rope_refusals(fn, kw, code):
    assert _rope(fn, **kw) == code


@pytest.mark.parametrize("fn", ["erase_rope", "erase_rope_backward"])
def test_rope_outputs_in_one_place(fn):
    same = (768, 256, 64)
    for kw in (dict(ko=R), dict(q=P, k=P, qo=P, ko=P, k_heads=4), dict(qo=Q), dict(ko=P)):
        assert _rope(fn, k_stride=same, ko_stride=same, **kw) == INVALID, kw
    assert _rope(fn, ko=R, batch=0) == erase.OK  # (nothing is written)


def test_rope_of_nothing():
    assert _rope(batch=0, q=None, k=None, qo=None, ko=None, table=None) == erase.OK
    assert _rope(seq=0, q=None, k=None, qo=None, ko=None, table=None) == erase.OK
    assert ops.lib().erase_rope(None, P, Q, R, S, None, P, None) == INVALID


def _norm(x=P, w=None, b=None, y=Q, mean=None, rstd=None, **kw):
    c = ops.NormConfig(4, 64, erase.BF16, 1e-5, 64, 64, 64, 64, 64)
    for name, v in kw.items():
        setattr(c, name, v)
    return ops.lib().erase_layer_norm(ctypes.byref(c), x, w, b, y, mean, rstd, None)


def test_norm_statistics_in_one_place():
    assert _norm(mean=R, rstd=R) == INVALID


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=2), INVALID), (dict(rows=-1), SHAPE), (dict(rows=1 << 31), SHAPE), (dict(cols=0), SHAPE),
    (dict(cols=16385), SHAPE), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID),
    (dict(x_ld=63), SHAPE), (dict(y_ld=63), SHAPE), (dict(x_ld=1 << 50), SHAPE), (dict(x=None), INVALID), (dict(y=None), INVALID),
    (dict(x=P + 1), INVALID), (dict(y=Q + 1), INVALID), (dict(dtype=0, x=P + 2), INVALID), (dict(w=P + 2), INVALID),
    (dict(b=P + 2), INVALID), (dict(mean=P + 1), INVALID), (dict(rstd=P + 2), INVALID), (dict(y=P, y_ld=128), INVALID)])
def test_layer_norm_refusals(kw, code):
    assert _norm(**kw) == code


def _norm_bwd(x=P, dy=Q, w=None, mean=S, rstd=S, res=None, dx=R, dw=S, db=None, scratch=P, short=0, **kw):
    c = ops.NormConfig(4, 64, erase.BF16, 1e-5, 64, 64, 64, 64, 64)
    for name, v in kw.items():
        setattr(c, name, v)
    n = ctypes.c_size_t(1)
    ops.lib().erase_layer_norm_backward_scratch_bytes(ctypes.byref(c), ctypes.byref(n))
    return ops.lib().erase_layer_norm_backward(ctypes.byref(c), x, dy, w, mean, rstd, res, dx, dw, db, scratch, n.value - short,
                                               None)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=2), INVALID), (dict(rows=-1), SHAPE), (dict(cols=0), SHAPE), (dict(cols=16385), SHAPE), (dict(x_ld=63), SHAPE),
    (dict(dy_ld=63), SHAPE), (dict(dx_ld=63), SHAPE), (dict(res=P, res_ld=63), SHAPE), (dict(x=None), INVALID),
    (dict(dy=None), INVALID), (dict(mean=None), INVALID), (dict(rstd=None), INVALID), (dict(x=P + 1), INVALID),
    (dict(dy=Q + 1), INVALID), (dict(res=P + 1), INVALID), (dict(dx=R + 1), INVALID), (dict(w=P + 2), INVALID),
    (dict(mean=P + 2), INVALID), (dict(rstd=P + 2), INVALID), (dict(dw=S + 2), INVALID), (dict(db=S + 2), INVALID),
    (dict(dw=S, db=S), INVALID), (dict(dx=P), INVALID), (dict(dx=Q, dx_ld=128), INVALID), (dict(res=R, res_ld=128), INVALID),
    (dict(scratch=None), WORKSPACE), (dict(scratch=P + 8), WORKSPACE), (dict(short=1), WORKSPACE)])
def test_layer_norm_backward_refusals(kw, code):
    assert _norm_bwd(**kw) == code


def test_layer_norm_of_nothing():
    assert _norm(rows=0, x=None, y=None) == erase.OK
    assert _norm_bwd(rows=0, x=None, dy=None, mean=None, rstd=None, dx=None, dw=None, scratch=None) == erase.OK
    assert _norm_bwd(dx=None, dw=None, scratch=None) == erase.OK  # nothing wanted
    assert ops.lib().erase_layer_norm(None, P, None, None, Q, None, None, None) == INVALID
    n = ctypes.c_size_t(0)
    assert ops.lib().erase_layer_norm_backward_scratch_bytes(None, ctypes.byref(n)) == INVALID
    c = ops.NormConfig(4, 64, erase.BF16, 1e-5, 64, 64, 64, 64, 64)
    assert ops.lib().erase_layer_norm_backward_scratch_bytes(ctypes.byref(c), None) == INVALID


def _drop(fn="erase_dropout", x=P, res=None, y=Q, step=None, **kw):
    c = ops.DropoutConfig(4, 64, erase.BF16, 0.5, 1, 2, 64, 64, 64)
    for name, v in kw.items():
        setattr(c, name, v)
    args = (x, res, y, step) if fn == "erase_dropout" else (x, y, step)
    return getattr(ops.lib(), fn)(ctypes.byref(c), *args, None)


@pytest.mark.parametrize("fn", ["erase_dropout", "erase_dropout_backward"])
@pytest.mark.parametrize("kw,code", [
    (dict(dtype=2), INVALID), (dict(p=-0.1), INVALID), (dict(p=1.1), INVALID), (dict(p=float("nan")), INVALID),
    (dict(rows=-1), SHAPE), (dict(rows=1 << 31), SHAPE), (dict(cols=-1), SHAPE), (dict(cols=1 << 31), SHAPE),
    (dict(rows=1 << 30, cols=1 << 30, x_ld=1 << 30, y_ld=1 << 30), SHAPE), (dict(x_ld=63), SHAPE), (dict(y_ld=63), SHAPE),
    (dict(x=None), INVALID), (dict(y=None), INVALID), (dict(x=P + 1), INVALID), (dict(y=Q + 1), INVALID),
    (dict(dtype=0, y=Q + 2), INVALID), (dict(step=P + 4), INVALID), (dict(y=P, y_ld=128), INVALID)])
def test_dropout_refusals(fn, kw, code):
    assert _drop(fn, **kw) == code


def test_dropout_residual_refusals_and_nothing():
    assert _drop(res=R + 1) == INVALID
    assert _drop(res=R, res_ld=63) == SHAPE
    assert _drop(res=Q, res_ld=128) == INVALID
    assert _drop(rows=0, x=None, y=None) == erase.OK and _drop(cols=0, x=None, y=None) == erase.OK
    assert ops.lib().erase_dropout(None, P, None, Q, None, None) == INVALID


def test_binding_refuses_host_tensors_and_types():
    import torch
    x = torch.zeros(4, 64)
    for call in (lambda: ops.layer_norm(x), lambda: ops.dropout(x, 0.5, 1), lambda: ops.dropout_backward(x, 0.5, 1),
                 lambda: ops.layer_norm(x.half()), lambda: ops.dropout(x.t(), 0.5, 1), lambda: ops.layer_norm(x[0]),
                 lambda: ops.layer_norm(x, torch.ones(63)), lambda: ops.layer_norm(x, torch.ones(64).double()),
                 lambda: ops.layer_norm_backward(x, x, None, x[:, 0], x[:, 0].contiguous()),
                 lambda: ops.layer_norm_backward(x[:3], x, None, torch.zeros(4), torch.zeros(4)),
                 lambda: ops.dropout(x, 0.5, -1), lambda: ops.dropout(x, 0.5, 1 << 64), lambda: ops.dropout(x, 0.5, 1, offset=-1),
                 lambda: ops.dropout(x, 0.5, 1, residual=x.bfloat16()), lambda: ops.dropout(x, 0.5, 1, step=torch.zeros(2)),
                 lambda: ops.rope_frequencies(64, scaling="cubic")):
        with pytest.raises(erase.EraseError):
            call()
    table = ops.RopeTable(ops.RopeSpec(32, 0, 10000.0, 1.0, 0.0, 32.0, 1.0), torch.zeros(17, dtype=torch.int64))
    q, k = torch.zeros(2, 3, 4, 32), torch.zeros(2, 3, 2, 32)
    for call in (lambda: ops.rope(q, k, table), lambda: ops.rope_backward(q, None, table), lambda: ops.rope(q[0], None, table),
                 lambda: ops.rope(q, k[:1], table), lambda: ops.rope(q, k, table, layout="both"),
                 lambda: ops.rope(q.transpose(2, 3), None, table)):
        with pytest.raises(erase.EraseError):
            call()
