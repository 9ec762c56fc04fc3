"""Cases of work for the operators around the token mixer: the norms before and after a block with its gate and residual scale
(`block_norm`, `block_join` and their backward passes), and the orthogonalised update of a matrix (`orthogonalize`,
`muon_update`).

Each case is one call of one operator on inputs as they stand in a training step or a forward of the block around the mixer.
With `own` false the operators are computed in their plain form, elementary torch operations in float32.
"""
import math

import torch

own = False

_DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
NS = (3.4445, -4.7750, 2.0315)          # the quintic's coefficients
EPS = 1e-5                              # of the norms
NS_EPS = 1e-7                           # beside the Frobenius norm
LR, DECAY, MOMENTUM = 0.02, 0.1, 0.95


# ------------------------------------------------------------------------------------------------- cases
def _block(name, op, B, N, C, dtype, res, norm, post, gate, scale, strided=False):
    """op: norm_fwd, norm_bwd, join_fwd, join_bwd.  res: type of the residual stream.  norm: layer (with bias) or rms (without).
    post: a norm behind the block too.  gate: none, token (sigmoid, one value per token and channel) or item (linear, one row per
    batch item).  scale: a residual scale per channel.  strided: branch and gate are slices of one wider projection."""
    return {"name": name, "op": op, "B": B, "N": N, "C": C, "dtype": dtype, "res": res, "norm": norm, "post": post, "gate": gate,
            "scale": scale, "strided": strided}


def _matrix(name, op, count, rows, cols, dtype):
    """op: orth (orthogonalize) or muon (muon_update: weights and momentum in float32, gradient in `dtype`)."""
    return {"name": name, "op": op, "count": count, "rows": rows, "cols": cols, "dtype": dtype}


def listed():
    return [
        # the smallest call: a few tokens of a wide model between two blocks, where only latency counts
        _block("join_fwd_4_tokens", "join_fwd", 1, 4, 4096, "bf16", "bf16", "rms", True, "token", False),
        # the norm before the first block over a batch of 2-D point clouds (8 heads of 16)
        _block("norm_fwd_mesh2d", "norm_fwd", 4, 65536, 128, "bf16", "bf16", "layer", False, "none", False),
        # its backward under float16 autocast, a width and a length that are multiples of nothing
        _block("norm_bwd_f16_odd", "norm_bwd", 4, 10007, 333, "f16", "f32", "layer", False, "none", False),
        # between two blocks over a million points (8 heads of 16), residual stream in float32
        _block("join_fwd_mesh3d_1m", "join_fwd", 1, 1048576, 128, "bf16", "f32", "layer", False, "none", True),
        # backward between two blocks for a padded batch conditioned per item (4 heads of 32; one gate row per item)
        _block("join_bwd_padded", "join_bwd", 32, 4096, 128, "bf16", "bf16", "layer", False, "item", False),
        # forward between two blocks of a wide model: norms on both sides, gate and branch out of one projection
        _block("join_fwd_wide", "join_fwd", 4, 4096, 4096, "bf16", "bf16", "rms", True, "token", True, True),
        # its backward
        _block("join_bwd_wide", "join_bwd", 4, 4096, 4096, "bf16", "bf16", "rms", True, "token", True, True),
        # backward in float32, as gradient checks and small regressions are run
        _block("join_bwd_f32", "join_bwd", 2, 9973, 200, "f32", "f32", "layer", True, "token", True),
        # the latent queries of one layer (8 heads of 256 latents 16 wide)
        _matrix("orth_latents", "orth", 8, 256, 16, "bf16"),
        # projection weights of a dozen blocks (two each, 8 heads of 16) in one update
        _matrix("muon_projections", "muon", 24, 128, 128, "f32"),
        # a tall matrix whose sides are multiples of nothing
        _matrix("orth_odd_tall", "orth", 1, 2601, 1003, "bf16"),
        # the square projections of one wide block (the largest case)
        _matrix("muon_wide", "muon", 2, 4096, 4096, "bf16"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    if rng.random() < 0.6:
        op = rng.choice(["norm_fwd", "norm_bwd", "join_fwd", "join_fwd", "join_bwd", "join_bwd"])
        dtype, res = rng.choice([("bf16", "bf16"), ("bf16", "bf16"), ("bf16", "f32"), ("f16", "f32"), ("f32", "f32")])
        C = _log_int(rng, 48, 8192)
        C = C if rng.random() < 0.25 else (C + 31) // 32 * 32
        rows = _log_int(rng, 1, max(2, min(1 << 20, (1 << 26) // C)))
        B = 1 if rows < 8 else rng.choice([1, 2, 4, 7])
        norm = rng.choice(["layer", "rms"])
        join = op.startswith("join")
        post = join and rng.random() < 0.6
        gate = rng.choice(["none", "token", "token", "item"]) if join else "none"
        scale = join and rng.random() < 0.5
        c = _block("", op, B, max(1, rows // B), C, dtype, res, norm, post, gate, scale, join and rng.random() < 0.3)
    else:
        op = rng.choice(["orth", "muon"])
        dtype = "bf16" if op == "orth" else rng.choice(["bf16", "f32", "f16"])
        if rng.random() < 0.5:                  # many small ones: latents, projections
            a, b = _log_int(rng, 16, 128), _log_int(rng, 16, 512)
            count = _log_int(rng, 1, 64)
        else:
            a = _log_int(rng, 128, 4096)
            b = _log_int(rng, a, min(8192, 4 * a, (1 << 24) // a))
            count = 1 if a * b > 1 << 22 else rng.choice([1, 1, 2, 3])
        if rng.random() < 0.7:
            a, b = (a + 15) // 16 * 16, (b + 15) // 16 * 16
        rows, cols = (a, b) if rng.random() < 0.5 else (b, a)
        c = _matrix("", op, count, rows, cols, dtype)
    del c["name"]
    return c


# ------------------------------------------------------------------------------------------------- inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _prepare_block(case, seed):
    g = _gen(seed)
    B, N, C = case["B"], case["N"], case["C"]
    T, R = _DTYPE[case["dtype"]], _DTYPE[case["res"]]

    def randn(*shape, scale=1.0, mean=0.0, dtype=torch.float32):
        return (torch.randn(*shape, device="cuda", generator=g) * scale + mean).to(dtype)

    def norm():
        # weights near one, biases near zero
        return {"w": randn(C, scale=0.1, mean=1.0), "b": randn(C, scale=0.1) if case["norm"] == "layer" else None}

    s = {"case": case, "pre": norm()}
    join, back = case["op"].startswith("join"), case["op"].endswith("bwd")
    # the residual stream: channels of unequal size, tokens of unequal size, a mean of its own per channel
    channel = randn(C, scale=0.5, mean=0.0).exp()
    x = randn(B, N, C) * channel * randn(B, N, 1, scale=0.3).exp() + 0.5 * randn(C)
    if join:
        wide = 2 * C if case["strided"] else C
        o = randn(B, N, wide, dtype=T)
        s["o"] = o[..., :C]
        s["post"] = norm() if case["post"] else None
        s["g"] = o[..., C:] if case["strided"] and case["gate"] == "token" else \
            randn(B, N, C, dtype=T) if case["gate"] == "token" else randn(B, C, mean=1.0, scale=0.5, dtype=T) if case["gate"] == "item" else None
        s["s"] = randn(C, scale=0.05, mean=0.2) if case["scale"] else None
    s["x"] = x.to(R)
    if back:
        del x
        if join:                                # the backward has the join's output in hand, and its statistics
            y, _, _, stats = _forward(s)
            s["x"] = y.to(R)
        else:
            stats = _forward(s)[3]
        s["stats"] = stats
        s["dh"] = randn(B, N, C, dtype=T)
        s["dy"] = randn(B, N, C, dtype=R) if join else None
    return s


def _prepare_matrix(case, seed):
    g = _gen(seed)
    count, rows, cols = case["count"], case["rows"], case["cols"]

    def randn(*shape):
        return torch.randn(*shape, device="cuda", generator=g)

    # a gradient: a few strong directions over noise, of the size gradients have
    r = max(1, min(rows, cols) // 16)
    grad = 1e-3 * (randn(count, rows, cols) + 2.0 * randn(count, rows, r) @ randn(count, r, cols) / math.sqrt(r))
    s = {"case": case, "g": grad.to(_DTYPE[case["dtype"]])}
    if case["op"] == "muon":
        s["w"] = randn(count, rows, cols) / math.sqrt(cols)
        s["m"] = 1e-3 * (randn(count, rows, cols) + 2.0 * randn(count, rows, r) @ randn(count, r, cols) / math.sqrt(r))
        # weights and momentum are updated into buffers of their own, so that a pass can be repeated
        s["w_out"], s["m_out"] = torch.empty_like(s["w"]), torch.empty_like(s["m"])
    return s


def prepare(case, seed):
    return (_prepare_matrix if case["op"] in ("orth", "muon") else _prepare_block)(case, seed)


# ------------------------------------------------------------------------------------------------- plain form
def _norm(x, kind, p):
    """x float32 [..., C] -> (normalised, mean, rstd, weighted)."""
    mean = x.mean(-1, keepdim=True) if kind == "layer" else torch.zeros_like(x[..., :1])
    d = x - mean
    rstd = 1.0 / torch.sqrt((d * d).mean(-1, keepdim=True) + EPS)
    hat = d * rstd
    out = hat * p["w"]
    return hat, mean, rstd, out if p["b"] is None else out + p["b"]


def _act(case, g):
    return 1.0 / (1.0 + torch.exp(-g)) if case["gate"] == "token" else g[:, None, :]


def _forward(s):
    """(y, h, None, stats [tokens, 4]: mean and rstd of the branch, mean and rstd of what the next norm sees), in float32."""
    case, x = s["case"], s["x"].float()
    zero = torch.zeros_like(x[..., :1])
    mean_o = rstd_o = zero
    if "o" in s:
        n = s["o"].float()
        if s["post"] is not None:
            _, mean_o, rstd_o, n = _norm(n, case["norm"], s["post"])
        if s["g"] is not None:
            n = n * _act(case, s["g"].float())
        if s["s"] is not None:
            n = n * s["s"]
        x = x + n
    _, mean, rstd, h = _norm(x, case["norm"], s["pre"])
    return x, h, None, torch.cat([mean_o, rstd_o, mean, rstd], -1).view(-1, 4)


def _norm_back(d, hat, rstd, kind, w):
    dw = d * w
    c = (dw * hat).mean(-1, keepdim=True)
    r = dw - hat * c
    if kind == "layer":
        r = r - dw.mean(-1, keepdim=True)
    return r * rstd


def _backward(s):
    case, kind = s["case"], s["case"]["norm"]
    T, R = _DTYPE[case["dtype"]], _DTYPE[case["res"]]
    st = s["stats"].view(case["B"], case["N"], 4)
    hat = (s["x"].float() - st[..., 2:3]) * st[..., 3:4]
    dh = s["dh"].float()
    rows = (0, 1)
    out = {"dw_pre": (dh * hat).sum(rows)}
    if s["pre"]["b"] is not None:
        out["db_pre"] = dh.sum(rows)
    dt = _norm_back(dh, hat, st[..., 3:4], kind, s["pre"]["w"])
    if s.get("dy") is not None:
        dt = dt + s["dy"].float()
    out["dx"] = dt.to(R)
    if "o" not in s:
        return out
    n = o = s["o"].float()
    if s["post"] is not None:
        o = (o - st[..., 0:1]) * st[..., 1:2]
        n = o * s["post"]["w"]
        n = n if s["post"]["b"] is None else n + s["post"]["b"]
    a = None if s["g"] is None else _act(case, s["g"].float())
    u = dt if a is None else dt * a
    if s["s"] is not None:
        out["ds"] = (u * n).sum(rows)
        u = u * s["s"]
    if a is not None:
        dg = dt * n if s["s"] is None else dt * n * s["s"]
        out["dg"] = (dg * a * (1.0 - a) if case["gate"] == "token" else dg.sum(1)).to(T)
    if s["post"] is not None:
        out["dw_post"] = (u * o).sum(rows)
        if s["post"]["b"] is not None:
            out["db_post"] = u.sum(rows)
        u = _norm_back(u, o, st[..., 1:2], kind, s["post"]["w"])
    out["do"] = u.to(T)
    return out


def _newton_schulz(u):
    """u float32 [..., R, C] -> the matrix after five steps of the quintic."""
    a, b, c = NS
    x = u / (torch.sqrt((u * u).sum((-2, -1), keepdim=True)) + NS_EPS)
    tall = x.shape[-2] > x.shape[-1]
    x = x.mT if tall else x
    for _ in range(5):
        gram = x @ x.mT
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return x.mT if tall else x


def _rho(case):
    return math.sqrt(max(1.0, case["rows"] / case["cols"]))


def _plain(s):
    case = s["case"]
    if case["op"] == "orth":
        return _newton_schulz(s["g"].float()).to(s["g"].dtype).contiguous()
    if case["op"] == "muon":
        g = s["g"].float()
        m = MOMENTUM * s["m"] + (1.0 - MOMENTUM) * g
        o = _newton_schulz(MOMENTUM * m + (1.0 - MOMENTUM) * g)
        return {"w": (1.0 - LR * DECAY) * s["w"] - LR * _rho(case) * o, "m": m}
    if case["op"].endswith("bwd"):
        return _backward(s)
    y, h, _, stats = _forward(s)
    out = {"h": h.to(_DTYPE[case["dtype"]]), "stats": stats}
    if case["op"] == "join_fwd":
        out["y"] = y.to(_DTYPE[case["res"]])
    return out


# ------------------------------------------------------------------------------------------------- the framework's calls
def _own(s):
    from paper_2508_12594_b200 import flare
    case = s["case"]
    if case["op"] == "orth":
        return flare.orthogonalize(s["g"], steps=5, coefficients=NS, eps=NS_EPS)
    if case["op"] == "muon":
        flare.muon_update(s["w"], s["m"], s["g"], lr=LR, momentum=MOMENTUM, weight_decay=DECAY, nesterov=True, update_scale=_rho(case),
                          steps=5, coefficients=NS, eps=NS_EPS, w_out=s["w_out"], m_out=s["m_out"])
        return {"w": s["w_out"], "m": s["m_out"]}
    T = _DTYPE[case["dtype"]]
    pre = flare.Norm(case["norm"], s["pre"]["w"], s["pre"]["b"], EPS)
    if case["op"] == "norm_fwd":
        h, stats = flare.block_norm(s["x"], pre, dtype=T)
        return {"h": h, "stats": stats}
    if case["op"] == "norm_bwd":
        r = flare.block_norm_backward(s["x"], s["stats"], s["dh"], pre)
        out = {"dx": r.dx, "dw_pre": r.dweight}
        if r.dbias is not None:
            out["db_pre"] = r.dbias
        return out
    post = None if s["post"] is None else flare.Norm(case["norm"], s["post"]["w"], s["post"]["b"], EPS)
    gate_kind = {"none": "none", "token": "sigmoid", "item": "linear"}[case["gate"]]
    if case["op"] == "join_fwd":
        y, h, stats = flare.block_join(s["x"], s["o"], post=post, pre=pre, gate=s["g"], gate_kind=gate_kind, scale=s["s"])
        return {"h": h, "stats": stats, "y": y}
    r = flare.block_join_backward(s["o"], s["x"], s["stats"], s["dy"], s["dh"], post=post, pre=pre, gate=s["g"], gate_kind=gate_kind, scale=s["s"])
    out = {"dw_pre": r.dpre_weight, "db_pre": r.dpre_bias, "dx": r.dx, "ds": r.dscale, "dg": r.dgate, "dw_post": r.dpost_weight,
           "db_post": r.dpost_bias, "do": r.dbranch}
    return {k: v for k, v in out.items() if v is not None}


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------------------------------------- work and exact values
def work(case):
    if case["op"] in ("orth", "muon"):
        n, R, C = case["count"], min(case["rows"], case["cols"]), max(case["rows"], case["cols"])
        e = 4 if case["dtype"] == "f32" else 2
        # a step: half of the symmetric X X^T, half of the symmetric square, one full product
        return {"bytes": n * R * C * (2 * e if case["op"] == "orth" else 16 + e), "flops": 5.0 * n * (R * R * C + R * R * R + 2.0 * R * R * C)}
    T, C = case["B"] * case["N"], case["C"]
    e, r = (4 if case[k] == "f32" else 2 for k in ("dtype", "res"))
    per = r + e                                                          # x and h, or x and dh
    join, back = case["op"].startswith("join"), case["op"].endswith("bwd")
    if back:
        per += r                                                         # dx
    if join:
        per += r + (e if not back else 0)                                # forward: y and the branch; backward: dy
        if back:                                                         # d branch; the branch itself where something needs it
            per += e + (e if case["post"] or case["scale"] or case["gate"] != "none" else 0)
        if case["gate"] == "token":
            per += e * (2 if back else 1)
    items = case["B"] * C * e * (2 if back else 1) if case["gate"] == "item" else 0
    return {"bytes": T * C * per + 16 * T + items, "flops": T * C * (40.0 if join and back else 12.0)}


def _exact_norm(v, kind, eps):
    if kind == "layer":
        var, mu = torch.var_mean(v, dim=-1, correction=0, keepdim=True)
    else:
        var, mu = v.pow(2).mean(-1, keepdim=True), torch.zeros_like(v[..., :1])
    return mu, (var + eps).rsqrt()


def _exact_block(case, seed):
    s = _prepare_block(case, seed)
    D = lambda t: None if t is None else t.double()  # noqa: E731
    B, N, C, kind = case["B"], case["N"], case["C"], case["norm"]
    w, b = D(s["pre"]["w"]), D(s["pre"]["b"])
    join = case["op"].startswith("join")
    o, g, sc = (D(s.get(k)) for k in ("o", "g", "s"))
    post = s.get("post")
    gate = None
    if g is not None:
        gate = torch.sigmoid(g) if case["gate"] == "token" else g.unsqueeze(1).expand(B, N, C)
    if case["op"].endswith("fwd"):
        v = D(s["x"])
        st_o = torch.zeros(B, N, 2, device="cuda", dtype=torch.float64)
        if join:
            branch = o
            if post is not None:
                mu, r = _exact_norm(o, kind, EPS)
                st_o = torch.cat([mu, r], -1)
                branch = torch.addcmul(D(post["b"]) if post["b"] is not None else torch.zeros(C, device="cuda", dtype=torch.float64), (o - mu) * r, D(post["w"]))
            for f in (gate, sc):
                branch = branch if f is None else branch * f
            v = v + branch
        mu, r = _exact_norm(v, kind, EPS)
        h = (v - mu) * r * w + (0.0 if b is None else b)
        out = {"h": h, "stats": torch.cat([st_o, mu, r], -1).reshape(-1, 4)}
        if join:
            out["y"] = v
        return out
    # backward: the vector-Jacobian products of the norm written out row by row
    st = D(s["stats"]).reshape(B, N, 4)
    dh, hat = D(s["dh"]), (D(s["x"]) - st[..., 2:3]) * st[..., 3:4]

    def pull(d, hat, rstd):
        centre = d - (d.sum(-1, keepdim=True) / C if kind == "layer" else 0.0)
        return rstd * (centre - hat * ((d * hat).sum(-1, keepdim=True) / C))

    out = {"dw_pre": torch.einsum("bnc,bnc->c", dh, hat)}
    if b is not None:
        out["db_pre"] = dh.sum((0, 1))
    dt = pull(dh * w, hat, st[..., 3:4])
    del hat, dh
    if s["dy"] is not None:
        dt = dt + D(s["dy"])
    out["dx"] = dt
    if not join:
        return out
    ohat, n = o, o
    if post is not None:
        ohat = (o - st[..., 0:1]) * st[..., 1:2]
        n = ohat * D(post["w"]) + (0.0 if post["b"] is None else D(post["b"]))
    factor = torch.ones(C, device="cuda", dtype=torch.float64) if sc is None else sc
    if sc is not None:
        out["ds"] = (dt * n * (1.0 if gate is None else gate)).sum((0, 1))
    if case["gate"] == "token":
        out["dg"] = dt * n * factor * gate * (1 - gate)
    elif case["gate"] == "item":
        out["dg"] = torch.einsum("bnc,bnc->bc", dt, n) * factor
    d = dt * factor * (1.0 if gate is None else gate)
    if post is not None:
        out["dw_post"] = torch.einsum("bnc,bnc->c", d, ohat)
        if post["b"] is not None:
            out["db_post"] = d.sum((0, 1))
        d = pull(d * D(post["w"]), ohat, st[..., 1:2])
    out["do"] = d
    return out


def exact(case, seed):
    if case["op"] not in ("orth", "muon"):
        return _exact_block(case, seed)
    s = _prepare_matrix(case, seed)
    a, b, c = NS
    g = s["g"].double()
    if case["op"] == "muon":
        m = torch.lerp(g, s["m"].double(), MOMENTUM)
        u = torch.lerp(g, m, MOMENTUM)
    else:
        u = g
    x = u / (torch.linalg.matrix_norm(u, keepdim=True) + NS_EPS)
    wide = case["rows"] <= case["cols"]
    for _ in range(5):                                                   # (X X^T) X = X (X^T X): the short side's matrix either way
        if wide:
            gram = torch.matmul(x, x.transpose(1, 2))
            x = a * x + b * torch.matmul(gram, x) + c * torch.matmul(torch.matmul(gram, gram), x)
        else:
            gram = torch.matmul(x.transpose(1, 2), x)
            x = a * x + b * torch.matmul(x, gram) + c * torch.matmul(x, torch.matmul(gram, gram))
    if case["op"] == "orth":
        return x
    return {"w": s["w"].double() * (1.0 - LR * DECAY) - LR * _rho(case) * x, "m": m}
