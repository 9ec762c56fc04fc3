"""Cases of work for what a model over tokens has at both ends of the mixer's blocks, and for dropout between them: the embedding
lookup and its gradient (`embed`, `embed_backward`), dropout from a counter-based generator (`dropout`, `dropout_backward`), and the
softmax cross entropy of a projection onto the vocabulary (`token_loss`, `token_loss_backward`).

Each case is one call (a training step of the loss: two) on inputs as a step or a scoring run has them.  With `own` false the
operators are computed in their plain form, elementary torch operations in float32.
"""
import math

import numpy as np
import torch

own = False

_DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_BYTES = {"f32": 4, "bf16": 2, "f16": 2}
M0, M1, W0, W1 = 0xD2511F53, 0xCD9E8D57, 0x9E3779B9, 0xBB67AE85      # Philox4x32: multipliers, key increments


# ------------------------------------------------------------------------------------------------- cases
def _embed(name, op, B, L, V, C, table, out, scale, positions, p, padding):
    """op: embed_fwd, embed_bwd.  table, out: types of the table (and its gradient) and of the rows.  positions: a table of positions
    too.  p: dropout.  padding: share of tokens that are none (-1)."""
    return {"name": name, "op": op, "B": B, "L": L, "V": V, "C": C, "table": table, "out": out, "scale": scale, "positions": positions,
            "p": p, "padding": padding}


def _drop(name, op, rows, C, dtype, res, p):
    """op: drop_fwd (with the residual's addition where `res` is a type), drop_bwd."""
    return {"name": name, "op": op, "rows": rows, "C": C, "dtype": dtype, "res": res, "p": p}


def _loss(name, op, rows, V, C, dtype, scale, padding, weights):
    """op: loss_fwd, loss_step (forward and gradients).  padding: share of rows without a label.  weights: every row has its own
    weight in the loss (else the mean over labelled rows)."""
    return {"name": name, "op": op, "rows": rows, "V": V, "C": C, "dtype": dtype, "scale": scale, "padding": padding, "weights": weights}


def listed():
    return [
        # the smallest call: one token on its way into a wide model
        _embed("embed_fwd_1_token", "embed_fwd", 1, 1, 32000, 1024, "bf16", "bf16", 32.0, False, 0.0, 0.0),
        # a padded batch of byte sequences (the long-sequence workload: 32 x 4096 tokens, 4 heads of 32), positions and dropout
        _embed("embed_fwd_padded", "embed_fwd", 32, 4096, 256, 128, "bf16", "bf16", 1.0, True, 0.1, 0.1),
        # its gradient: few rows, thousands of tokens each
        _embed("embed_bwd_padded", "embed_bwd", 32, 4096, 256, 128, "bf16", "bf16", 1.0, True, 0.1, 0.1),
        # gradient of a large vocabulary's table in float32 from bfloat16 activations: most rows are met by no token
        _embed("embed_bwd_vocab", "embed_bwd", 4, 4099, 50021, 1000, "f32", "bf16", 31.6, False, 0.0, 0.02),
        # behind a block over a million points (8 heads of 16), onto a residual stream in float32
        _drop("drop_fwd_mesh3d_1m", "drop_fwd", 1048576, 128, "bf16", "f32", 0.1),
        # backward under float16 autocast, a width and a length that are multiples of nothing
        _drop("drop_bwd_f16_odd", "drop_bwd", 40028, 333, "f16", None, 0.25),
        # scoring one token against a vocabulary
        _loss("loss_fwd_1_token", "loss_fwd", 1, 32000, 1024, "bf16", 1.0, 0.0, False),
        # scoring a ragged batch in float16
        _loss("loss_fwd_f16_ragged", "loss_fwd", 5003, 50021, 1000, "f16", 1.0, 0.3, False),
        # training step of the padded byte sequences
        _loss("loss_step_padded", "loss_step", 131072, 256, 128, "bf16", 1.0, 0.1, False),
        # training step in float32, odd sizes, a weight for every row
        _loss("loss_step_f32", "loss_step", 1999, 10007, 200, "f32", 0.5, 0.1, True),
        # training step of a small model with a tied vocabulary
        _loss("loss_step_vocab", "loss_step", 4096, 32000, 512, "bf16", 1.0, 0.02, False),
        # the largest: a wide model's loss over a large vocabulary
        _loss("loss_step_wide", "loss_step", 8192, 128256, 1024, "bf16", 1.0, 0.02, False),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    C = _log_int(rng, lo, hi)
    return C if rng.random() < 0.25 else (C + 31) // 32 * 32


def draw(rng):
    kind = rng.random()
    if kind < 0.35:
        table, out = rng.choice([("bf16", "bf16"), ("bf16", "bf16"), ("f32", "bf16"), ("f32", "f16"), ("f16", "f16"), ("bf16", "f32"), ("f32", "f32")])
        C = _width(rng, 16, 4096)
        V = _log_int(rng, 16, min(131072, (1 << 27) // C))
        L = _log_int(rng, 1, min(65536, (1 << 26) // C))
        B = rng.choice([1, 2, 4, 7, 32]) if L * C <= 1 << 20 else 1
        c = _embed("", rng.choice(["embed_fwd", "embed_bwd"]), B, L, V, C, table, out, rng.choice([1.0, round(math.sqrt(C), 3)]), rng.random() < 0.4,
                   rng.choice([0.0, 0.1, 0.1, 0.5]), rng.choice([0.0, 0.1]))
    elif kind < 0.6:
        dtype, res = rng.choice([("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32"), ("f32", "f32"), ("bf16", None)])
        op = rng.choice(["drop_fwd", "drop_bwd"])
        C = _width(rng, 16, 8192)
        c = _drop("", op, _log_int(rng, 1, min(1 << 20, (1 << 27) // C)), C, dtype, res if op == "drop_fwd" else None, round(rng.uniform(0.02, 0.6), 3))
    else:
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        most = 1 << (36 if dtype == "f32" else 38)
        C = _width(rng, 32, 4096)
        V = _log_int(rng, 2, min(131072, (1 << 27) // C))
        rows = _log_int(rng, 1, max(2, min(65536, most // (C * V), (1 << 30) // V)))
        c = _loss("", rng.choice(["loss_fwd", "loss_step", "loss_step"]), rows, V, C, dtype, rng.choice([1.0, 1.0, 0.5]), rng.choice([0.0, 0.1, 0.3]),
                  rng.random() < 0.4)
    del c["name"]
    return c


# ------------------------------------------------------------------------------------------------- inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _tokens(g, n, V, padding):
    """Token numbers as texts have them: a few are met all the time, most hardly ever."""
    u = torch.rand(n, device="cuda", generator=g, dtype=torch.float64)
    rank = (torch.exp(u * math.log(V + 1.0)) - 1.0).long().clamp_(0, V - 1)
    t = (rank * 7919 + 13) % V                                    # (frequent ones are not next to each other)
    if padding > 0:
        t = torch.where(torch.rand(n, device="cuda", generator=g) < padding, torch.full_like(t, -1), t)
    return t


def prepare(case, seed):
    g = _gen(seed)
    s = {"case": case}

    def randn(*shape, scale=1.0, dtype=torch.float32):
        return (torch.randn(*shape, device="cuda", generator=g) * scale).to(dtype)

    if case["op"].startswith("embed"):
        T, O = _DTYPE[case["table"]], _DTYPE[case["out"]]
        B, L, V, C = case["B"], case["L"], case["V"], case["C"]
        s["tokens"] = _tokens(g, B * L, V, case["padding"]).view(B, L)
        s["table"] = randn(V, C, scale=1.0 / case["scale"], dtype=T)
        s["positions"] = randn(L, C, scale=0.3, dtype=T) if case["positions"] else None
        if case["op"] == "embed_bwd":
            s["dy"] = randn(B, L, C, scale=0.02, dtype=O)
    elif case["op"].startswith("drop"):
        T = _DTYPE[case["dtype"]]
        s["x"] = randn(case["rows"], case["C"], dtype=T)
        if case["res"]:
            s["residual"] = randn(case["rows"], case["C"], dtype=_DTYPE[case["res"]])
    else:
        T, rows, V, C = _DTYPE[case["dtype"]], case["rows"], case["V"], case["C"]
        s["x"] = randn(rows, C, dtype=T)                           # behind a norm
        s["w"] = randn(V, C, scale=2.0 / (math.sqrt(C) * case["scale"]), dtype=T)
        labels = _tokens(g, rows, V, case["padding"])
        if rows > 1:                                               # some rows have learned their label
            sure = (torch.rand(rows, device="cuda", generator=g) < 0.3) & (labels >= 0)
            s["x"][sure] = (s["x"][sure].float() + 3.0 * case["scale"] * s["w"][labels[sure]].float()).to(T)
        else:
            labels.clamp_(min=0)
        s["labels"] = torch.where(labels < 0, torch.full_like(labels, -100), labels)
        if case["weights"]:
            s["dloss"] = torch.rand(rows, device="cuda", generator=g) * (2.0 / rows)
        else:
            s["dloss"] = 1.0 / max(1, int((s["labels"] >= 0).sum()))
    s["seed"], s["offset"] = (seed * 0x9E3779B97F4A7C15 + 12345) % (1 << 63), seed * 3 + 5
    return s


# ------------------------------------------------------------------------------------------------- plain forms
def _mulhilo(a, m):
    """High and low word of the product of 32-bit numbers held in int64 (its 64 bits wrap to the right ones)."""
    p = a * m
    return (p >> 32) & 0xFFFFFFFF, p & 0xFFFFFFFF


def _keep_plain(rows, C, p, seed, offset, device):
    """Factors of dropout [rows, C]: 0, or what makes up for those."""
    thr = int(round(p * 65536))
    groups = (C + 7) // 8
    c0 = torch.arange(groups, device=device, dtype=torch.int64).expand(rows, groups)
    c1 = torch.arange(rows, device=device, dtype=torch.int64)[:, None].expand(rows, groups)
    c2, c3 = torch.full_like(c0, offset & 0xFFFFFFFF), torch.full_like(c0, offset >> 32)
    k0, k1 = seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF
    m0, m1 = M0, M1
    for _ in range(10):
        h0, l0 = _mulhilo(c0, m0)
        h1, l1 = _mulhilo(c2, m1)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + W0) & 0xFFFFFFFF, (k1 + W1) & 0xFFFFFFFF
    words = torch.stack([c0, c1, c2, c3], -1)
    u = torch.stack([words & 0xFFFF, words >> 16], -1).view(rows, groups * 8)[:, :C]
    return (u >= thr).float() * (65536.0 / (65536 - thr) if thr < 65536 else 0.0)


def _drop_plain(x, case, s):
    """x [rows, C] float32, rows in pieces for the generator's sake."""
    if round(case["p"] * 65536) == 0:
        return x
    n, C = x.shape
    return x * _keep_plain(n, C, case["p"], s["seed"], s["offset"], x.device)


def _embed_plain(s):
    c = s["case"]
    t, V, C, O = s["tokens"].reshape(-1), c["V"], c["C"], _DTYPE[c["out"]]
    there = (t >= 0) & (t < V)
    if c["op"] == "embed_fwd":
        y = s["table"][t.clamp(0, V - 1)].float() * c["scale"] * there[:, None]
        if s["positions"] is not None:
            y = (y.view(c["B"], c["L"], C) + s["positions"].float()).view(-1, C)
        return {"y": _drop_plain(y, c, s).to(O).view(c["B"], c["L"], C)}
    d = _drop_plain(s["dy"].float().view(-1, C), c, s)
    table = torch.zeros(V, C, device=d.device).index_add_(0, t[there], d[there]) * c["scale"]
    r = {"dtable": table.to(_DTYPE[c["table"]])}
    if c["positions"]:
        r["dpositions"] = d.view(c["B"], c["L"], C).sum(0).to(_DTYPE[c["table"]])
    return r


def _dropout_plain(s):
    c = s["case"]
    y = _drop_plain(s["x"].float(), c, s)
    if c["res"]:
        y = y + s["residual"].float()
    return {"y": y.to(_DTYPE[c["res"] or c["dtype"]])}


def _loss_plain(s):
    c = s["case"]
    x, w, labels, T = s["x"].float(), s["w"].float(), s["labels"], _DTYPE[c["dtype"]]
    there = (labels >= 0) & (labels < c["V"])
    at = labels.clamp(0, c["V"] - 1)[:, None]
    logits = (x @ w.T).mul_(c["scale"])
    top = logits.max(1, keepdim=True).values
    chosen = logits.gather(1, at)
    lse = top + logits.sub(top).exp_().sum(1, keepdim=True).log()
    loss = torch.where(there, (lse - chosen)[:, 0], 0.0)
    if c["op"] == "loss_fwd":
        return {"loss": loss, "lse": torch.where(there, lse[:, 0], 0.0)}
    g = logits.sub_(lse).exp_()
    g.scatter_add_(1, at, torch.full_like(lse, -1.0))
    g.mul_(torch.where(there, s["dloss"], 0.0)[:, None]).mul_(c["scale"])
    return {"loss": loss, "dx": (g @ w).to(T), "dw": (g.T @ x).to(T)}


# ------------------------------------------------------------------------------------------------- run
def run(state):
    s, c = state, state["case"]
    if not own:
        return _embed_plain(s) if c["op"].startswith("embed") else _dropout_plain(s) if c["op"].startswith("drop") else _loss_plain(s)
    from paper_2508_12594_b200 import flare

    if c["op"].startswith("loss"):
        loss, lse = flare.token_loss(s["x"], s["w"], s["labels"], scale=c["scale"])
        if c["op"] == "loss_fwd":
            return {"loss": loss, "lse": lse}
        g = flare.token_loss_backward(s["x"], s["w"], s["labels"], lse, s["dloss"], scale=c["scale"])
        return {"loss": loss, "dx": g.dx, "dw": g.dw}
    drop = flare.Drop(c["p"], s["seed"], s["offset"]) if c["p"] > 0 else None
    if c["op"] == "embed_fwd":
        return {"y": flare.embed(s["tokens"], s["table"], positions=s["positions"], scale=c["scale"], drop=drop, dtype=_DTYPE[c["out"]])}
    if c["op"] == "embed_bwd":
        g = flare.embed_backward(s["tokens"], s["dy"], c["V"], positions=c["L"] if c["positions"] else 0, scale=c["scale"], drop=drop,
                                 dtype=_DTYPE[c["table"]])
        return {"dtable": g.dtable, "dpositions": g.dpositions} if c["positions"] else {"dtable": g.dtable}
    if c["op"] == "drop_fwd":
        return {"y": flare.dropout(s["x"], drop, residual=s.get("residual"))}
    return {"y": flare.dropout_backward(s["x"], drop)}


def work(case):
    c = case
    if c["op"].startswith("embed"):
        n, C, t, o = c["B"] * c["L"], c["C"], _BYTES[c["table"]], _BYTES[c["out"]]
        rows = min(n, c["V"])                                      # of the table that tokens can meet
        pos = c["L"] * C * t if c["positions"] else 0
        moved = rows * C * t if c["op"] == "embed_fwd" else c["V"] * C * t
        return {"bytes": n * 8 + n * C * o + moved + pos, "flops": 2 * n * C}
    if c["op"].startswith("drop"):
        t = _BYTES[c["dtype"]]
        r = _BYTES[c["res"]] if c["res"] else 0
        return {"bytes": c["rows"] * c["C"] * (t + (2 * r if r else t)), "flops": 2 * c["rows"] * c["C"]}
    t, n, V, C = _BYTES[c["dtype"]], c["rows"], c["V"], c["C"]
    labelled = n * (1.0 - c["padding"])
    step = c["op"] == "loss_step"
    return {"bytes": (n * C + V * C) * t * (2 if step else 1) + n * 12, "flops": int((6 if step else 2) * labelled * V * C)}


# ------------------------------------------------------------------------------------------------- from the definition, in 64 bits
def _philox(counter, key):
    """Philox4x32-10 over arrays of uint64 that hold 32-bit words."""
    low = np.uint64(0xFFFFFFFF)
    c0, c1, c2, c3 = counter
    k0, k1 = key
    for _ in range(10):
        a, b = c0 * np.uint64(M0), c2 * np.uint64(M1)
        c0, c1, c2, c3 = (b >> np.uint64(32)) ^ c1 ^ np.uint64(k0), b & low, (a >> np.uint64(32)) ^ c3 ^ np.uint64(k1), a & low
        k0, k1 = (k0 + W0) & 0xFFFFFFFF, (k1 + W1) & 0xFFFFFFFF
    return c0, c1, c2, c3


def _factors(rows, C, p, seed, offset):
    """Row by row blocks of dropout's factors, float64 on the GPU."""
    thr = round(p * 65536)
    if thr == 0:
        return torch.ones(rows, C, dtype=torch.float64, device="cuda")
    groups = -(-C // 8)
    out = torch.empty(rows, C, dtype=torch.bool)
    step = max(1, (1 << 22) // groups)
    for r0 in range(0, rows, step):
        r1 = min(rows, r0 + step)
        n = (r1 - r0) * groups
        col = np.tile(np.arange(groups, dtype=np.uint64), r1 - r0)
        row = np.repeat(np.arange(r0, r1, dtype=np.uint64), groups)
        words = _philox((col, row, np.full(n, offset % (1 << 32), np.uint64), np.full(n, offset >> 32, np.uint64)), (seed % (1 << 32), seed >> 32))
        bits = np.empty((n, 8), np.uint16)
        for k, w in enumerate(words):
            bits[:, 2 * k] = (w & np.uint64(0xFFFF)).astype(np.uint16)
            bits[:, 2 * k + 1] = (w >> np.uint64(16)).astype(np.uint16)
        out[r0:r1] = torch.from_numpy(bits.reshape(r1 - r0, groups * 8)[:, :C] >= thr)
    keep = 65536.0 / (65536 - thr) if thr < 65536 else 0.0
    return out.cuda().double().mul_(keep)


def exact(case, seed):
    s, c = prepare(case, seed), case
    if c["op"].startswith("drop"):
        y = s["x"].double() * _factors(c["rows"], c["C"], c["p"], s["seed"], s["offset"])
        return {"y": y + s["residual"].double() if c["res"] else y}
    if c["op"].startswith("embed"):
        n, C, V = c["B"] * c["L"], c["C"], c["V"]
        f = _factors(n, C, c["p"], s["seed"], s["offset"])
        t = s["tokens"].reshape(-1)
        if c["op"] == "embed_fwd":
            rows = torch.cat([s["table"].double() * c["scale"], torch.zeros(1, C, dtype=torch.float64, device="cuda")])
            y = torch.index_select(rows, 0, torch.where(t < 0, V, t)).view(c["B"], c["L"], C)
            if c["positions"]:
                y = y + s["positions"].double()[None]
            return {"y": y * f.view(c["B"], c["L"], C)}
        d = s["dy"].double().view(n, C) * f
        del f
        dpos = torch.stack([d.view(c["B"], c["L"], C)[b] for b in range(c["B"])]).sum(0) if c["positions"] else None
        order = torch.argsort(t, stable=True)                       # sums of runs of equal tokens as differences of running sums
        ends = torch.bincount(t + 1, minlength=V + 1).cumsum(0)
        runs = torch.cat([torch.zeros(1, C, dtype=torch.float64, device="cuda"), d[order].cumsum(0)])
        r = {"dtable": (runs[ends[1:]] - runs[ends[:-1]]) * c["scale"]}
        if c["positions"]:
            r["dpositions"] = dpos
        return r
    if 8.0 * c["rows"] * c["V"] * c["C"] > 2e16:                    # (beyond some ten seconds in 64 bits)
        return None
    x, w, labels, V = s["x"].double(), s["w"].double(), s["labels"], c["V"]
    n, step = c["rows"], max(1, (1 << 28) // V)
    dloss = s["dloss"].double() if c["weights"] else torch.full((n,), s["dloss"], dtype=torch.float64, device="cuda")
    loss, dx, dw = torch.zeros(n, dtype=torch.float64, device="cuda"), torch.zeros_like(x), torch.zeros_like(w)
    lse = torch.zeros_like(loss)
    for r0 in range(0, n, step):
        at = torch.nonzero(labels[r0:r0 + step] >= 0)[:, 0] + r0
        if at.numel() == 0:
            continue
        logits = c["scale"] * torch.matmul(x[at], w.mT)
        logp = torch.log_softmax(logits, dim=1)
        mark = torch.nn.functional.one_hot(labels[at], V) if V * at.numel() < 1 << 26 else None
        lse[at] = torch.logsumexp(logits, 1)
        loss[at] = -torch.take_along_dim(logp, labels[at][:, None], 1)[:, 0]
        if c["op"] == "loss_step":
            p = logp.exp()
            if mark is not None:
                p = p - mark
            else:
                p[torch.arange(at.numel(), device="cuda"), labels[at]] -= 1.0
            p *= (c["scale"] * dloss[at])[:, None]
            dx[at] = p @ w
            dw += p.mT @ x[at]
    return {"loss": loss, "lse": lse} if c["op"] == "loss_fwd" else {"loss": loss, "dx": dx, "dw": dw}
