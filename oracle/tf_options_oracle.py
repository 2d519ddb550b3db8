"""CPU oracle of the transformer step with options: rotary positions, layer
norms with learned weight and bias, dropout of the two branches, in the blocks
of transformer_oracle.py.

TEST INFRASTRUCTURE ONLY.  Nothing in the product path imports, links or runs
this module.  It shares no code with the HIP library; the masks and the
frequencies are those of ops_oracle.py, the gradients torch's autograd on the
CPU, the update transformer_oracle's Adam.

    n1 = norm(a0; g1, b1);  [q | k | v] = n1 Wqkv^T;  q, k turned by position t
    o  = causal softmax attention per head;  a1 = a0 + drop(o Wo^T)
    n2 = norm(a1; g2, b2);  z = a1 + drop(gelu(n2 W1^T) W2^T)
    loss_b = mean of -log softmax(norm(z; g3, b3) Wh^T)[next token]

drop draws from key `dropout_seed`, row = position, offset ((2 block + branch)
<< 40) + step number.  ``emulate_bf16`` rounds what the GPU stores in bf16: the
value of a stored activation, and the gradient that is stored beside it.
"""
from __future__ import annotations

import math

import numpy as np
import torch

from . import ops_oracle as oo
from .erase_oracle import adam_update

__all__ = ["tf_step"]


class _Stored(torch.autograd.Function):
    """A tensor kept in bf16 whose gradient (when `grad`) is kept in bf16 too."""

    @staticmethod
    def forward(ctx, x, grad):
        ctx.grad = grad
        return x.to(torch.bfloat16).to(x.dtype)

    @staticmethod
    def backward(ctx, g):
        return (g.to(torch.bfloat16).to(g.dtype) if ctx.grad else g), None


def _norm(cfg, p, x, i):
    if cfg.get("norm", "rms") == "layer":
        m = x.mean(-1, keepdim=True)
        r = 1.0 / torch.sqrt(((x - m) ** 2).mean(-1, keepdim=True) + cfg.get("norm_eps", 1e-5))
        return (x - m) * r * p["g%d" % i] + p["b%d" % i]
    return x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-6)


def _turn(cfg, x):
    """x [B][T][H][dh] turned by its position."""
    r = cfg.get("rope")
    if r is None:
        return x
    kw = {k: v for k, v in r.items() if k != "layout"}
    f, amp = oo.rope_frequencies(**kw)
    n = len(f)
    th = np.arange(x.shape[1])[:, None, None] * f
    c, s = (torch.from_numpy(amp * fn(th)).to(x.dtype) for fn in (np.cos, np.sin))
    if r.get("layout", "half") == "half":
        a, b = x[..., :n], x[..., n:2 * n]
        return torch.cat([a * c - b * s, b * c + a * s, x[..., 2 * n:]], -1)
    a, b = x[..., 0:2 * n:2], x[..., 1:2 * n:2]
    return torch.cat([torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2), x[..., 2 * n:]], -1)


def _block(cfg, p, a0, b, step, stored):
    """(z, head input) of block b."""
    B, T, H = cfg["batch"], cfg["seq"], cfg["heads"]
    N, d = a0.shape
    drop = cfg.get("dropout", 0.0)

    def branch(x, i):
        if drop == 0.0:
            return x
        kept, scale = oo.dropout_kept(N, d, drop, cfg.get("dropout_seed", 0), ((2 * b + i) << 40) + step)
        return stored(x, True) * torch.from_numpy(kept * scale).to(x.dtype)

    w = {k: stored(p[k], False) for k in ("wqkv", "wo", "w1", "w2")}
    n1 = stored(_norm(cfg, p, a0, 1), True)
    qkv = stored(n1 @ w["wqkv"].t(), True).view(B, T, 3, H, d // H)
    q, k = (stored(_turn(cfg, qkv[:, :, i]), True).transpose(1, 2) for i in range(2))
    v = qkv[:, :, 2].transpose(1, 2)
    s = (q @ k.transpose(-1, -2)) / math.sqrt(d // H)
    s = s.masked_fill(torch.ones((T, T), dtype=torch.bool).triu(1), -math.inf)
    o = stored((torch.softmax(s, -1) @ v).transpose(1, 2).reshape(N, d), True)
    a1 = stored(a0 + branch(o @ w["wo"].t(), 0), True)
    n2 = stored(_norm(cfg, p, a1, 2), True)
    u = n2 @ w["w1"].t()
    g = stored(torch.nn.functional.gelu(u, approximate="tanh"), False)
    z = stored(a1 + branch(g @ w["w2"].t(), 1), True)
    return z, stored(_norm(cfg, p, z, 3), True)


def tf_step(cfg: dict, params: list, m: list, v: list, t: int, tokens, emulate_bf16: bool = False, dtype=np.float64) -> dict:
    """One training step; arguments and result as transformer_oracle.tf_step."""
    stored = _Stored.apply if emulate_bf16 else (lambda x, grad: x)
    tokens = torch.from_numpy(np.asarray(tokens)).long()
    inp, tgt = tokens[:, :-1].reshape(-1), tokens[:, 1:].reshape(-1)
    lam, ad, t1 = cfg.get("lam", 1.0), cfg["adam"], t + 1
    out = {"losses": [], "grads": [], "params": [], "m": [], "v": [], "t": t1}
    a0 = None
    for b, block in enumerate(params):
        p = {k: torch.from_numpy(np.asarray(x, dtype=dtype)).requires_grad_() for k, x in block.items()}
        a0 = stored(p["emb"], False)[inp] if b == 0 else a0.detach()
        z, hn = _block(cfg, p, a0, b, t1, stored)
        loss = torch.nn.functional.cross_entropy(hn @ stored(p["wh"], False).t(), tgt)
        grads = torch.autograd.grad(lam * loss, list(p.values()))
        out["losses"].append(float(loss.detach()))
        g = {k: x.numpy() for k, x in zip(p, grads)}
        new = {k: adam_update(np.asarray(block[k], dtype=dtype), np.asarray(m[b][k], dtype=dtype),
                              np.asarray(v[b][k], dtype=dtype), g[k], t1, **ad) for k in g}
        out["grads"].append(g)
        for i, name in enumerate(("params", "m", "v")):
            out[name].append({k: new[k][i] for k in new})
        a0 = z
    return out
