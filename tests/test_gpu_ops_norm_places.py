"""Where a layer norm's dx is stored and what that leaves the same."""
import numpy as np
import pytest

from paper_2608_18469_amd import erase_ops as ops
from tests.test_gpu_ops import _dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("R,C", [(20, 300), (33, 512), (40, 5), (300, 515), (768, 64), (129, 2050), (500, 4097), (65, 12345),
                                 (769, 512)])
def test_gradients_wherever_dx_is_stored(dtype, R, C):
    """dx has the same bits apart, over dy and over the residual's gradient; so have
    dw and db but with dx over dy, where they may be summed in another order, the
    same for every such call."""
    import torch
    rng = np.random.Generator(np.random.PCG64(R + C))
    mk = lambda: _dev(rng.normal(size=(R, C)), dtype)[0]
    x, dy, res = mk(), mk(), mk()
    w = _dev(rng.normal(size=C), "f32")[0]
    _, m, r = ops.layer_norm(x, w)
    print("[norm backward, places]", dtype, R, C, flush=True)
    want = ops.layer_norm_backward(dy, x, w, m, r, residual=res)
    again = ops.layer_norm_backward(dy, x, w, m, r, residual=(q := res.clone()), out=(q, None, None))
    none = ops.layer_norm_backward(dy, x, w, m, r, residual=res, need_input=False)
    for got in (again, none):
        assert got[0] is None or torch.equal(got[0], want[0])
        assert torch.equal(got[1], want[1]) and torch.equal(got[2], want[2])
    over = [ops.layer_norm_backward(d := dy.clone(), x, w, m, r, residual=res, out=(d, None, None)) for _ in range(3)]
    for got in over:
        assert torch.equal(got[0], want[0])
        assert torch.equal(got[1], over[0][1]) and torch.equal(got[2], over[0][2])
    d = dy.clone()
    only = ops.layer_norm_backward(d, x, w, m, r, residual=res, need_weight=False, out=(d, None, None))
    assert only[1] is None and torch.equal(only[0], want[0]) and torch.equal(only[2], over[0][2])
