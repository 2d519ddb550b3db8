"""Workloads for timing the operators of a transformer block around its GEMMs
and its attention: rotary positions, layer norm and dropout, each forward and
backward.

A case is a plain dict.  ``listed()`` gives the fixed ones, ``draw(rng)`` one
more of the same ranges, ``prepare(case, seed)`` what a program holds before
the call, ``run(state)`` one pass (plain torch operations in 32 bits, or the
library's entry points when ``own`` is set), ``work(case)`` the bytes and
operations a pass cannot do without, ``exact(case, seed)`` the same outputs
from the definitions in 64 bits.
"""
import math

import numpy as np
import torch

own = False

EPS = 1e-5  # of the layer norms
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------
def listed():
    return [
        # one new token for each of 32 sequences, far into their contexts, grouped key heads: latency
        dict(name="rope_token", kind="rope", dtype="bf16", batch=32, seq=1, q_heads=8, k_heads=2, head_dim=64, rot_dim=64,
             layout="half", scaling="none", factor=1.0, length=0, positions="far", packed=False, start=0),
        # the small-transformer training shape: queries and keys inside one packed projection
        dict(name="rope_train", kind="rope", dtype="bf16", batch=16, seq=1024, q_heads=8, k_heads=8, head_dim=64,
             rot_dim=64, layout="half", scaling="none", factor=1.0, length=0, positions="none", packed=True, start=0),
        # a long context in one sequence: adjacent pairs in half of each head, frequencies scaled by parts
        dict(name="rope_long", kind="rope", dtype="bf16", batch=1, seq=32768, q_heads=32, k_heads=8, head_dim=128,
             rot_dim=64, layout="interleaved", scaling="by_parts", factor=8.0, length=16384, positions="none", packed=False,
             start=98304),
        # the gradient of a ragged fp32 batch of packed documents (positions start again), 48 of 80 columns rotated
        dict(name="rope_backward_ragged", kind="rope_backward", dtype="f32", batch=3, seq=777, q_heads=5, k_heads=1,
             head_dim=80, rot_dim=48, layout="half", scaling="linear", factor=4.0, length=0, positions="restart",
             packed=False, start=0),
        # a handful of rows (latency)
        dict(name="norm_few_rows", kind="norm", dtype="bf16", rows=16, cols=512, bias=True),
        # every position of the small-transformer training shape
        dict(name="norm_train", kind="norm", dtype="bf16", rows=16384, cols=512, bias=True),
        # fp32 rows of the CTR input's odd width
        dict(name="norm_odd_width", kind="norm", dtype="f32", rows=3001, cols=1677, bias=True),
        # the backward pass of the training shape, with the residual path's gradient added
        dict(name="norm_backward_train", kind="norm_backward", dtype="bf16", rows=16384, cols=512, bias=True, residual=True),
        # the widest model the transformer step takes
        dict(name="norm_backward_wide", kind="norm_backward", dtype="bf16", rows=16384, cols=4096, bias=True,
             residual=False),
        # a small fp32 activation of odd width (latency)
        dict(name="dropout_small", kind="dropout", dtype="f32", rows=64, cols=401, p=0.5, residual=False),
        # a branch of a block joining the residual stream in training
        dict(name="dropout_add_train", kind="dropout", dtype="bf16", rows=16384, cols=512, p=0.1, residual=True),
        # the gradient into the branch of the widest model
        dict(name="dropout_backward_wide", kind="dropout_backward", dtype="bf16", rows=16384, cols=4096, p=0.1,
             residual=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rope", "rope_backward", "norm", "norm_backward", "dropout", "dropout_backward"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind.startswith("rope"):
        head_dim = rng.choice([32, 64, 64, 80, 96, 128, 128, 192, 256])
        rot_dim = rng.choice([head_dim, head_dim, head_dim // 2, 2 * rng.randint(1, head_dim // 2)])
        k_heads = rng.choice([1, 2, 4, 8])
        q_heads = k_heads * rng.choice([1, 2, 4, 5])
        most = (1 << 27) // ((q_heads + k_heads) * head_dim * (2 if dtype == "f32" else 1))  # tokens
        seq = 1 if rng.random() < 0.25 else _log_int(rng, 2, min(most, 32768))
        batch = _log_int(rng, 1, max(1, min(64, most // seq)))
        scaling = rng.choice(["none", "none", "linear", "ntk", "by_parts"])
        return dict(kind=kind, dtype=dtype, batch=batch, seq=seq, q_heads=q_heads, k_heads=k_heads, head_dim=head_dim,
                    rot_dim=rot_dim, layout=rng.choice(["half", "interleaved"]), scaling=scaling,
                    factor=1.0 if scaling == "none" else rng.choice([2.0, 4.0, 8.0, 32.0]),
                    length=rng.choice([2048, 4096, 8192]) if scaling == "by_parts" else 0,
                    positions=rng.choice(["none", "far", "restart"]), packed=kind == "rope" and rng.random() < 0.4,
                    start=rng.choice([0, 0, _log_int(rng, 1, 1 << 20)]))
    if kind.startswith("norm"):
        cols = _log_int(rng, 16, 8192)
        if rng.random() < 0.5:
            cols = max(64, cols // 64 * 64)
        rows = _log_int(rng, 1, (1 << 25) // cols)
        return dict(kind=kind, dtype=dtype, rows=rows, cols=cols, bias=rng.random() < 0.8,
                    **({"residual": rng.random() < 0.5} if kind == "norm_backward" else {}))
    cols = _log_int(rng, 8, 16384)
    if rng.random() < 0.5:
        cols = cols // 8 * 8
    rows = _log_int(rng, 1, (1 << 25) // cols)
    return dict(kind=kind, dtype=dtype, rows=rows, cols=cols, p=rng.choice([0.0, 0.1, 0.1, 0.2, 0.5, rng.random()]),
                residual=kind == "dropout" and rng.random() < 0.6)


# ---------------------------------------------------------------------------
# inputs, from the seed alone
# ---------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _rope_inputs(case, seed):
    """(q [B][T][Hq][D], k [B][T][Hk][D], positions int32 [B][T] or None)."""
    g = _gen(seed)
    B, T, Hq, Hk, D = (case[k] for k in ("batch", "seq", "q_heads", "k_heads", "head_dim"))
    scale = 1e-4 if case["kind"] == "rope_backward" else 1.0  # gradients are small
    dt = TYPES[case["dtype"]]
    if case["packed"]:  # queries | keys | values of one projection
        x = torch.randn((B, T, (Hq + 2 * Hk) * D), generator=g, device="cuda").to(dt)
        q = x[..., :Hq * D].unflatten(-1, (Hq, D))
        k = x[..., Hq * D:(Hq + Hk) * D].unflatten(-1, (Hk, D))
    else:
        q = (torch.randn((B, T, Hq, D), generator=g, device="cuda") * scale).to(dt)
        k = (torch.randn((B, T, Hk, D), generator=g, device="cuda") * scale).to(dt)
    pos = None
    t = torch.arange(T, device="cuda")
    if case["positions"] == "far":  # a position of its own for each sequence, up to 2^17
        first = torch.randint(0, 1 << 17, (B, 1), generator=g, device="cuda")
        pos = (first + t).to(torch.int32)
    elif case["positions"] == "restart":  # documents of random lengths, each from 0
        cut = torch.rand((B, T), generator=g, device="cuda") < 4.0 / T
        begin = torch.cummax(torch.where(cut, t, torch.zeros_like(t)), dim=1).values
        pos = (t - begin).to(torch.int32)
    return q, k, pos


def _norm_inputs(case, seed):
    """(x, w, b or None, dy, res or None): a residual stream with a few strong columns, and its gradients."""
    g = _gen(seed)
    R, C, dt = case["rows"], case["cols"], TYPES[case["dtype"]]
    col = 1.0 + 7.0 * (torch.rand(C, generator=g, device="cuda") < 0.01)
    x = ((torch.randn((R, C), generator=g, device="cuda") + 0.3) * col).to(dt)
    w = 1.0 + 0.2 * torch.randn(C, generator=g, device="cuda")
    b = 0.1 * torch.randn(C, generator=g, device="cuda") if case["bias"] else None
    dy = res = None
    if case["kind"] == "norm_backward":
        dy = (torch.randn((R, C), generator=g, device="cuda") * 1e-3).to(dt)
        if case["residual"]:
            res = (torch.randn((R, C), generator=g, device="cuda") * 1e-3).to(dt)
    return x, w, b, dy, res


def _dropout_inputs(case, seed):
    """(x or its gradient, residual or None, generator seed, offset)."""
    g = _gen(seed)
    R, C, dt = case["rows"], case["cols"], TYPES[case["dtype"]]
    x = torch.randn((R, C), generator=g, device="cuda").to(dt)
    res = torch.randn((R, C), generator=g, device="cuda").to(dt) if case["residual"] else None
    return x, res, (int(seed) * 0x9E3779B97F4A7C15 + 12345) % (1 << 64), ((int(seed) << 33) + 7) % (1 << 64)


# ---------------------------------------------------------------------------
# what a program holds before the call
# ---------------------------------------------------------------------------
def prepare(case, seed):
    kind = case["kind"]
    s = {"kind": kind, "case": dict(case)}
    if kind.startswith("rope"):
        q, k, pos = _rope_inputs(case, seed)
        s.update(q=q, k=k, pos=pos)
        if own:
            from paper_2608_18469_amd import erase_ops
            s["table"] = erase_ops.rope_table(case["rot_dim"], scaling=case["scaling"], factor=case["factor"],
                                              original_length=case["length"])
            s["out"] = (torch.empty(q.shape, dtype=q.dtype, device="cuda"), torch.empty(k.shape, dtype=k.dtype, device="cuda"))
        else:
            freq, amp = _freq_plain(case)
            s.update(freq=freq, amp=amp)
        return s
    if kind.startswith("norm"):
        x, w, b, dy, res = _norm_inputs(case, seed)
        s.update(x=x, w=w, b=b, dy=dy, res=res)
        if kind == "norm_backward":  # the forward pass's statistics
            xd = x.double()
            mean = xd.mean(1)
            s["rstd"] = (1.0 / torch.sqrt((xd - mean[:, None]).square().mean(1) + EPS)).float()
            s["mean"] = mean.float()
        if own:
            from paper_2608_18469_amd import erase_ops
            if kind == "norm":
                s["out"] = (torch.empty_like(x), torch.empty(case["rows"], device="cuda"), torch.empty(case["rows"], device="cuda"))
            else:
                s["out"] = (torch.empty_like(x), torch.empty_like(w), torch.empty_like(b) if b is not None else None)
                s["scratch"] = erase_ops.layer_norm_backward_scratch(x)
        return s
    x, res, gen, offset = _dropout_inputs(case, seed)
    s.update(x=x, res=res, gen=gen, offset=offset)
    if own:
        s["out"] = torch.empty_like(x)
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s):
    from paper_2608_18469_amd import erase_ops as ops
    c, kind = s["case"], s["kind"]
    if kind == "rope":
        return ops.rope(s["q"], s["k"], s["table"], positions=s["pos"], start=c["start"], layout=c["layout"], out=s["out"])
    if kind == "rope_backward":
        return ops.rope_backward(s["q"], s["k"], s["table"], positions=s["pos"], start=c["start"], layout=c["layout"],
                                 out=s["out"])
    if kind == "norm":
        return ops.layer_norm(s["x"], s["w"], s["b"], eps=EPS, out=s["out"])
    if kind == "norm_backward":
        return ops.layer_norm_backward(s["dy"], s["x"], s["w"], s["mean"], s["rstd"], residual=s["res"],
                                       need_bias=s["b"] is not None, out=s["out"], scratch=s["scratch"])
    if kind == "dropout":
        return ops.dropout(s["x"], c["p"], s["gen"], offset=s["offset"], residual=s["res"], out=s["out"])
    return ops.dropout_backward(s["x"], c["p"], s["gen"], offset=s["offset"], out=s["out"])


def _freq_plain(case):
    """Angle per position of every pair (64 bits), and the amplitude of the rotation."""
    r, s, base = case["rot_dim"], case["factor"], 10000.0
    if case["scaling"] == "ntk" and r > 2:
        base = base * s ** (r / (r - 2))
    f = base ** (-torch.arange(0, r, 2, dtype=torch.float64, device="cuda") / r)
    if case["scaling"] == "linear":
        f = f / s
    if case["scaling"] == "by_parts":  # kept above 32 turns in the original length, divided by s below 1
        turns = case["length"] * f / (2 * math.pi)
        keep = ((turns - 1.0) / 31.0).clamp(0, 1)
        return f * keep + f / s * (1 - keep), 0.1 * math.log(s) + 1
    return f, 1.0


def _run_plain(s):
    c, kind = s["case"], s["kind"]
    if kind.startswith("rope"):
        r, T = c["rot_dim"], c["seq"]
        pos = s["pos"] if s["pos"] is not None else torch.arange(c["start"], c["start"] + T, device="cuda")[None]
        angle = pos.double()[..., None] * s["freq"]
        cos = (torch.cos(angle) * s["amp"]).float()[:, :, None]
        sin = (torch.sin(angle) * s["amp"]).float()[:, :, None]
        if kind == "rope_backward":
            sin = -sin
        out = []
        for x in (s["q"], s["k"]):
            y = x.float()
            if c["layout"] == "half":
                a, b = y[..., :r // 2], y[..., r // 2:r]
                y = torch.cat([a * cos - b * sin, b * cos + a * sin, y[..., r:]], -1)
            else:
                a, b = y[..., 0:r:2], y[..., 1:r:2]
                rot = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
                y = torch.cat([rot, y[..., r:]], -1)
            out.append(y.to(x.dtype))
        return tuple(out)
    if kind == "norm":
        x = s["x"].float()
        mean = x.mean(1, keepdim=True)
        d = x - mean
        rstd = 1.0 / torch.sqrt((d * d).mean(1, keepdim=True) + EPS)
        y = d * rstd * s["w"]
        if s["b"] is not None:
            y = y + s["b"]
        return y.to(s["x"].dtype), mean[:, 0], rstd[:, 0]
    if kind == "norm_backward":
        x, dy, rstd = s["x"].float(), s["dy"].float(), s["rstd"][:, None]
        h = (x - s["mean"][:, None]) * rstd
        g = dy * s["w"]
        dx = rstd * (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True))
        if s["res"] is not None:
            dx = dx + s["res"].float()
        return dx.to(s["x"].dtype), (dy * h).sum(0), dy.sum(0) if s["b"] is not None else None
    R, C = c["rows"], c["cols"]
    limit = min(65536, int(math.floor(c["p"] * 65536 + 0.5)))
    y = torch.where(_halves_plain(R, C, s["gen"], s["offset"]) >= limit,
                    s["x"].float() * (65536.0 / (65536 - limit) if limit < 65536 else 0.0), 0.0)
    if s["res"] is not None:
        y = y + s["res"].float()
    return y.to(s["x"].dtype)


def _halves_plain(R, C, seed, offset):
    """16 random bits for each element of [R][C]: Philox4x32-10 (Salmon, Moraes, Dror, Shaw 2011), key = seed,
    counter = (column / 8, row, offset); eight 16-bit halves of a result serve eight columns, low halves first."""
    M, groups = 0xFFFFFFFF, -(-C // 8)
    x0 = torch.arange(groups, device="cuda").expand(R, groups)
    x1 = torch.arange(R, device="cuda")[:, None].expand(R, groups)
    x2, x3 = torch.full_like(x0, offset & M), torch.full_like(x0, offset >> 32)
    k0, k1 = seed & M, seed >> 32
    for _ in range(10):
        p, q = x0 * 0xD2511F53, x2 * 0xCD9E8D57  # modulo 2^64
        x0, x1, x2, x3 = ((q >> 32) & M) ^ x1 ^ k0, q & M, ((p >> 32) & M) ^ x3 ^ k1, p & M
        k0, k1 = (k0 + 0x9E3779B9) & M, (k1 + 0xBB67AE85) & M
    words = torch.stack([x0, x1, x2, x3], -1)
    return torch.stack([words & 0xFFFF, words >> 16], -1).reshape(R, 8 * groups)[:, :C]


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    kind, size = case["kind"], 2.0 if case["dtype"] == "bf16" else 4.0
    if kind.startswith("rope"):
        tokens, heads = float(case["batch"] * case["seq"]), case["q_heads"] + case["k_heads"]
        ids = 4.0 * tokens if case["positions"] != "none" else 0.0
        return {"bytes": 2.0 * tokens * heads * case["head_dim"] * size + ids, "flops": 3.0 * tokens * heads * case["rot_dim"]}
    n, c = float(case["rows"]) * case["cols"], float(case["cols"])
    vectors = 2.0 if case.get("bias") else 1.0
    if kind == "norm":
        return {"bytes": 2.0 * n * size + 4.0 * vectors * c + 8.0 * case["rows"], "flops": 8.0 * n}
    if kind == "norm_backward":
        return {"bytes": (4.0 if case["residual"] else 3.0) * n * size + 4.0 * c + 4.0 * vectors * c + 8.0 * case["rows"],
                "flops": 14.0 * n}
    return {"bytes": (3.0 if case["residual"] else 2.0) * n * size, "flops": 2.0 * n}


# ---------------------------------------------------------------------------
# the same outputs in 64 bits
# ---------------------------------------------------------------------------
def exact(case, seed):
    kind = case["kind"]
    if kind.startswith("rope"):
        q, k, pos = _rope_inputs(case, seed)
        r, s = case["rot_dim"], case["factor"]
        freq, amp = [], 1.0
        for i in range(r // 2):
            f = math.pow(10000.0, -2.0 * i / r)
            if case["scaling"] == "linear":
                f /= s
            elif case["scaling"] == "ntk" and r > 2:
                f *= math.pow(s, -2.0 * i / (r - 2))
            elif case["scaling"] == "by_parts":
                share = min(1.0, max(0.0, (case["length"] * f / math.tau - 1.0) / 31.0))
                f *= share + (1.0 - share) / s
                amp = 1.0 + 0.1 * math.log(s)
            freq.append(f)
        if pos is None:
            pos = case["start"] + torch.arange(case["seq"], device="cuda").repeat(case["batch"], 1)
        theta = pos.to(torch.float64)[:, :, None] * torch.tensor(freq, dtype=torch.float64, device="cuda")
        if kind == "rope_backward":
            theta = -theta
        turn = torch.polar(torch.full_like(theta, amp), theta)[:, :, None]
        out = []
        for x in (q, k):
            y = x.double().contiguous()
            rot = y[..., :r]
            pairs = rot.unflatten(-1, (2, r // 2)).transpose(-1, -2) if case["layout"] == "half" else rot.unflatten(-1, (r // 2, 2))
            z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
            y[..., :r] = (z.transpose(-1, -2) if case["layout"] == "half" else z).flatten(-2)
            out.append(y)
        return tuple(out)
    if kind.startswith("norm"):
        x, w, b, dy, res = (None if t is None else t.double() for t in _norm_inputs(case, seed))
        var, mean = torch.var_mean(x, dim=1, correction=0, keepdim=True)
        rstd = torch.rsqrt(var + EPS)
        hat = (x - mean) * rstd
        if kind == "norm":
            return hat * w + (0.0 if b is None else b), mean.squeeze(1), rstd.squeeze(1)
        # the gradient of sum(dy * (hat w + b)) through hat(x)
        g = dy * w
        n = case["cols"]
        dx = (rstd / n) * (n * g - g.sum(1, keepdim=True) - hat * (g * hat).sum(1, keepdim=True))
        return dx if res is None else dx + res, torch.einsum("rc,rc->c", dy, hat), None if b is None else dy.sum(0)
    x, res, gen, offset = _dropout_inputs(case, seed)
    limit = min(65536, int(math.floor(case["p"] * 65536 + 0.5)))
    keep = torch.from_numpy(_halves_numpy(case["rows"], case["cols"], gen, offset) >= limit).cuda()
    y = torch.zeros_like(x, dtype=torch.float64)
    y[keep] = x.double()[keep] * 65536.0 / (65536 - limit) if limit < 65536 else 0.0
    return y if res is None else y + res.double()


def _halves_numpy(R, C, seed, offset):
    """The 16-bit values of _halves_plain, in unsigned host arithmetic: one array of four words per counter."""
    G = -(-C // 8)
    u64, low, by = np.uint64, np.uint64(0xFFFFFFFF), np.uint64(32)
    w = np.empty((4, R, G), u64)
    w[0], w[1] = np.arange(G, dtype=u64), np.arange(R, dtype=u64)[:, None]
    w[2], w[3] = u64(offset & 0xFFFFFFFF), u64(offset >> 32)
    for i in range(10):
        key = [u64(((seed & 0xFFFFFFFF) + i * 0x9E3779B9) & 0xFFFFFFFF), u64(((seed >> 32) + i * 0xBB67AE85) & 0xFFFFFFFF)]
        a, b = w[0] * u64(0xD2511F53), w[2] * u64(0xCD9E8D57)
        w[0], w[2] = (b >> by) ^ w[1] ^ key[0], (a >> by) ^ w[3] ^ key[1]
        w[1], w[3] = b & low, a & low
    return w.astype("<u4").transpose(1, 2, 0).copy().view("<u2").reshape(R, 8 * G)[:, :C].astype(np.int32)
