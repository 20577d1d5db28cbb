"""Workloads of the output end of a language model in training: layer normalisation with its backward
pass, the vocabulary head with its softmax cross-entropy and gradients without a logits matrix, and
distillation from a teacher's top logits.

`listed` names the cases, `draw` makes more of the same ranges, `prepare` builds a case's inputs on the
GPU from a seed, `run` makes one pass through the operator: in plain torch operations in 32 bits, or,
with the module variable `own` set, through the library.  `exact` evaluates the definitions in 64 bits
and `work` counts the bytes and operations a pass cannot do without.
"""
import math

import torch

own = False

LN_EPS = 1e-5


def listed():
    return [
        # the rows of one time step of a small batch: what a normalisation costs when only latency counts
        {"name": "ln_fwd_step", "op": "ln_fwd", "rows": 64, "cols": 1024, "pitch": 1024, "beta": True},
        # activations of the wide MLP layer (batch 4096, 12288 features)
        {"name": "ln_fwd_wide", "op": "ln_fwd", "rows": 4096, "cols": 12288, "pitch": 12288, "beta": True},
        # all T*B = 20*2048 projected outputs of the LSTM layer, backward
        {"name": "ln_bwd_lstm", "op": "ln_bwd", "rows": 40960, "cols": 1024, "pitch": 1024, "beta": True},
        # odd row count and odd width in pitched rows, no shift vector, backward
        {"name": "ln_bwd_odd", "op": "ln_bwd", "rows": 2047, "cols": 8191, "pitch": 8192, "beta": False},
        # a small classifier head: training step whose products are all launch-bound
        {"name": "lce_small", "op": "lce", "N": 64, "V": 1000, "H": 512, "grads": "both", "row_block": 0, "pad": 0.0},
        # the 12288 -> 32000 head of the large MLP at batch 4096, loss and both gradients
        {"name": "lce_head", "op": "lce", "N": 4096, "V": 32000, "H": 12288, "grads": "both", "row_block": 0, "pad": 0.0},
        # full softmax over a word-level vocabulary of 793471 from 1024 projected features; a tenth of the rows is padding
        {"name": "lce_words", "op": "lce", "N": 1024, "V": 793471, "H": 1024, "grads": "both", "row_block": 0, "pad": 0.1},
        # evaluation: losses only, odd sizes
        {"name": "lce_eval", "op": "lce", "N": 2500, "V": 50001, "H": 2048, "grads": "none", "row_block": 0, "pad": 0.05},
        # a small classifier distilled from 8 teacher logits per row
        {"name": "distill_small", "op": "distill", "B": 64, "C": 1000, "pitch": 1000, "K": 8, "tau": 2.0, "pad": 0.0},
        # the logits of the large MLP's head, 64 teacher logits per row
        {"name": "distill_head", "op": "distill", "B": 4096, "C": 32000, "pitch": 32000, "K": 64, "tau": 2.0, "pad": 0.0},
        # rows too long for one SM's shared memory
        {"name": "distill_words", "op": "distill", "B": 512, "C": 793471, "pitch": 793472, "K": 128, "tau": 1.0, "pad": 0.1},
        # odd class count, ragged teacher lists (padded entries, some rows with none at all)
        {"name": "distill_ragged", "op": "distill", "B": 2001, "C": 20011, "pitch": 20016, "K": 20, "tau": 4.0, "pad": 0.3},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["ln_fwd", "ln_bwd", "lce", "distill"])
    if op in ("ln_fwd", "ln_bwd"):
        cols = _log(rng, 8, 20000)
        rows = min(_log(rng, 1, 60000), 50000000 // cols)
        pitch = rng.choice([cols, (cols + 7) // 8 * 8, (cols + 7) // 8 * 8 + 8])
        return {"op": op, "rows": rows, "cols": cols, "pitch": pitch, "beta": rng.random() < 0.7}
    if op == "lce":
        H = 8 * _log(rng, 8, 1536)
        V = min(_log(rng, 64, 800000), 800000000 // H)
        N = min(_log(rng, 1, 4096), 800000000 // V, int(1.5e12 / (float(V) * H)))
        N = max(1, N)
        return {"op": op, "N": N, "V": V, "H": H, "grads": rng.choice(["both", "both", "dx", "none"]),
                "row_block": rng.choice([0, 0, 512]), "pad": rng.choice([0.0, 0.1])}
    C = _log(rng, 16, 800000)
    B = max(1, min(_log(rng, 1, 5000), 200000000 // C))
    K = min(_log(rng, 1, 256), C)
    return {"op": op, "B": B, "C": C, "pitch": rng.choice([C, (C + 7) // 8 * 8, (C + 7) // 8 * 8 + 8]), "K": K,
            "tau": rng.choice([1.0, 2.0, 4.0]), "pad": rng.choice([0.0, 0.3])}


def _rows(rows, cols, pitch, make):
    """A [rows, cols] FP16 view of a [rows, pitch] buffer."""
    buf = torch.zeros(rows, pitch, dtype=torch.float16, device="cuda")
    buf[:, :cols] = make
    return buf[:, :cols]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape, scale=1.0, shift=0.0):
        return (torch.randn(*shape, generator=g, device="cuda") * scale + shift).half()

    s = {"case": case}
    if case["op"] in ("ln_fwd", "ln_bwd"):
        rows, cols, pitch = case["rows"], case["cols"], case["pitch"]
        s["x"] = _rows(rows, cols, pitch, normal(rows, cols, scale=1.5, shift=0.25))
        s["gamma"] = normal(cols, scale=0.2, shift=1.0)
        s["beta"] = normal(cols, scale=0.2) if case["beta"] else None
        if case["op"] == "ln_bwd":
            s["dy"] = _rows(rows, cols, pitch, normal(rows, cols, scale=0.125))
            x = s["x"].float()
            s["mean"] = x.mean(1)
            s["rstd"] = torch.rsqrt(x.var(1, unbiased=False) + LN_EPS)
        return s
    if case["op"] == "lce":
        N, V, H = case["N"], case["V"], case["H"]
        s["S"] = 2.0 ** (2 + N.bit_length())      # the factor on a row's gradient, S / N, is between 4 and 8
        s["x"] = normal(N, H)
        s["W"] = normal(V, H, scale=2.0 / math.sqrt(H))
        y = (V * torch.rand(N, generator=g, device="cuda") ** 3).int().clamp_(max=V - 1)      # frequent words first
        s["y"] = torch.where(torch.rand(N, generator=g, device="cuda") < case["pad"], torch.full_like(y, -1), y)
        return s
    B, C, K = case["B"], case["C"], case["K"]
    s["S"] = 2.0 ** (2 + B.bit_length())
    s["z"] = _rows(B, C, case["pitch"], normal(B, C, scale=2.0))
    step = max(1, C // K)      # distinct classes in every row, spread over the whole range
    first = torch.randint(0, step, (B, K), generator=g, device="cuda")
    idx = (torch.arange(K, device="cuda") * step + first).int()
    s["t"] = torch.sort(normal(B, K, scale=2.0, shift=6.0), dim=1, descending=True).values.contiguous()
    gone = torch.rand(B, K, generator=g, device="cuda") < case["pad"]
    gone |= torch.rand(B, 1, generator=g, device="cuda") < case["pad"] / 4
    s["idx"] = torch.where(gone, torch.full_like(idx, -1), idx)
    return s


# ---------------------------------------------------------------- the plain forms, 32 bits

def _plain_ln_fwd(s):
    x = s["x"].float()
    mean = x.mean(1)
    d = x - mean[:, None]
    rstd = 1.0 / torch.sqrt((d * d).mean(1) + LN_EPS)
    y = d * rstd[:, None] * s["gamma"].float()
    if s["beta"] is not None:
        y = y + s["beta"].float()
    return {"y": y.half(), "mean": mean, "rstd": rstd}


def _plain_ln_bwd(s):
    dy = s["dy"].float()
    h = (s["x"].float() - s["mean"][:, None]) * s["rstd"][:, None]
    gy = dy * s["gamma"].float()
    dx = (gy - gy.mean(1)[:, None] - h * (gy * h).mean(1)[:, None]) * s["rstd"][:, None]
    out = {"dx": dx.half(), "dgamma": (dy * h).sum(0).half()}
    if s["beta"] is not None:
        out["dbeta"] = dy.sum(0).half()
    return out


def _plain_lce(s):
    x, W, y, N = s["x"].float(), s["W"].float(), s["y"].long(), s["case"]["N"]
    z = x @ W.t()
    z = z - z.max(1).values[:, None]
    e = torch.exp(z)
    total = e.sum(1)
    live = y >= 0
    at = y.clamp(min=0)[:, None]
    row_loss = torch.where(live, torch.log(total) - z.gather(1, at)[:, 0], torch.zeros_like(total))
    out = {"row_loss": row_loss, "loss": (row_loss.double().sum() / N).float()}
    if s["case"]["grads"] == "none":
        return out
    del z
    e *= (live / total)[:, None]
    e.scatter_add_(1, at, -live.float()[:, None])
    c = s["S"] / N
    out["dx"] = ((e @ W) * c).half()
    if s["case"]["grads"] == "both":
        out["dW"] = ((e.t() @ x) * c).half()
    return out


def _plain_distill(s):
    tau, B = s["case"]["tau"], s["case"]["B"]
    z = s["z"].float() / tau
    z = z - z.max(1).values[:, None]
    logp = z - torch.log(torch.exp(z).sum(1))[:, None]
    valid = s["idx"] >= 0
    live = valid.any(1)
    t = torch.where(valid, s["t"].float() / tau, torch.full_like(s["t"], -math.inf, dtype=torch.float32))
    top = torch.where(live, t.max(1).values, torch.zeros_like(t[:, 0]))
    w = torch.exp(t - top[:, None])
    norm = torch.where(live, w.sum(1), torch.ones_like(top))
    q = w / norm[:, None]
    logq = t - top[:, None] - torch.log(norm)[:, None]
    at = s["idx"].clamp(min=0).long()
    terms = torch.where(q > 0, q * (logq - logp.gather(1, at)), torch.zeros_like(q))
    row_loss = terms.sum(1) * (tau * tau)
    d = torch.exp(logp) * live[:, None]
    d.scatter_add_(1, at, -q)
    return {"dz": (d * (tau * s["S"] / B)).half(), "row_loss": row_loss, "loss": (row_loss.double().sum() / B).float()}


# ---------------------------------------------------------------- the library's calls

def _buffers(s, make):
    """The output and scratch tensors a program keeps from one pass to the next."""
    if "buffers" not in s:
        s["buffers"] = make()
    return s["buffers"]


def _own_ln_fwd(s):
    from paper_1710_03740_b200 import binding as b
    c = s["case"]
    rows, cols = c["rows"], c["cols"]
    o = _buffers(s, lambda: {"y": torch.empty(rows, c["pitch"], dtype=torch.float16, device="cuda")[:, :cols],
                             "mean": torch.empty(rows, dtype=torch.float32, device="cuda"),
                             "rstd": torch.empty(rows, dtype=torch.float32, device="cuda")})
    b.mpt_layernorm_forward(rows, cols, s["x"], c["pitch"], s["gamma"], s["beta"], LN_EPS, o["y"], c["pitch"], o["mean"], o["rstd"])
    return o


def _own_ln_bwd(s):
    from paper_1710_03740_b200 import binding as b
    c = s["case"]
    rows, cols = c["rows"], c["cols"]

    def make():
        o = {"dx": torch.empty(rows, c["pitch"], dtype=torch.float16, device="cuda")[:, :cols],
             "dgamma": torch.empty(cols, dtype=torch.float16, device="cuda")}
        if s["beta"] is not None:
            o["dbeta"] = torch.empty(cols, dtype=torch.float16, device="cuda")
        return o, torch.empty(b.mpt_layernorm_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    o, ws = _buffers(s, make)
    b.mpt_layernorm_backward(rows, cols, s["dy"], c["pitch"], s["x"], c["pitch"], s["gamma"], s["mean"], s["rstd"], o["dx"],
                             c["pitch"], o["dgamma"], o.get("dbeta"), ws)
    return o


def _own_lce(s):
    from paper_1710_03740_b200 import binding as b
    c = s["case"]
    N, V, H = c["N"], c["V"], c["H"]

    def make():
        o = {"row_loss": torch.empty(N, dtype=torch.float32, device="cuda"), "loss": torch.empty((), dtype=torch.float32, device="cuda")}
        if c["grads"] != "none":
            o["dx"] = torch.empty(N, H, dtype=torch.float16, device="cuda")
        if c["grads"] == "both":
            o["dW"] = torch.empty(V, H, dtype=torch.float16, device="cuda")
        nbytes = b.mpt_linear_ce_workspace_bytes(N, V, H, "dx" in o, "dW" in o, c["row_block"])
        return o, torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    o, ws = _buffers(s, make)
    b.mpt_linear_ce(N, V, H, s["x"], H, s["W"], H, s["y"], s["S"], o["row_loss"], o["loss"], o.get("dx"), H, o.get("dW"), H, ws,
                    row_block=c["row_block"])
    return o


def _own_distill(s):
    from paper_1710_03740_b200 import binding as b
    c = s["case"]
    B, C, K = c["B"], c["C"], c["K"]
    o = _buffers(s, lambda: {"dz": torch.empty(B, c["pitch"], dtype=torch.float16, device="cuda")[:, :C],
                             "row_loss": torch.empty(B, dtype=torch.float32, device="cuda"),
                             "loss": torch.empty((), dtype=torch.float32, device="cuda")})
    b.mpt_distill_topk(s["z"], c["pitch"], B, C, s["t"], s["idx"], K, K, c["tau"], s["S"], o["dz"], c["pitch"], o["row_loss"], o["loss"])
    return o


def run(state):
    op = state["case"]["op"]
    if own:
        return {"ln_fwd": _own_ln_fwd, "ln_bwd": _own_ln_bwd, "lce": _own_lce, "distill": _own_distill}[op](state)
    return {"ln_fwd": _plain_ln_fwd, "ln_bwd": _plain_ln_bwd, "lce": _plain_lce, "distill": _plain_distill}[op](state)


# ---------------------------------------------------------------- 64 bits, and what a pass has to move

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("ln_fwd", "ln_bwd"):
        x = s["x"].double()
        if case["op"] == "ln_fwd":
            var, mean = torch.var_mean(x, 1, correction=0)
            y = torch.nn.functional.layer_norm(x, (case["cols"],), s["gamma"].double(),
                                               None if s["beta"] is None else s["beta"].double(), LN_EPS)
            return {"y": y, "mean": mean, "rstd": (var + LN_EPS).rsqrt()}
        # the statistics are inputs of the backward pass: differentiate through them as the forward pass defines them
        r, m, n = s["rstd"].double()[:, None], s["mean"].double()[:, None], case["cols"]
        h, dy = (x - m) * r, s["dy"].double()
        dh = dy * s["gamma"].double()
        dvar = (dh * (x - m)).sum(1, keepdim=True) * (-0.5) * r ** 3
        dmean = -(dh * r).sum(1, keepdim=True)      # the variance's own term vanishes: deviations from the mean sum to zero
        out = {"dx": dh * r + dvar * 2.0 * (x - m) / n + dmean / n, "dgamma": torch.einsum("rc,rc->c", dy, h)}
        if s["beta"] is not None:
            out["dbeta"] = torch.einsum("rc->c", dy)
        return out
    if case["op"] == "lce":
        x, W, N = s["x"].double(), s["W"].double(), case["N"]
        row_loss = torch.zeros(N, dtype=torch.float64, device="cuda")
        dx = torch.zeros_like(x) if case["grads"] != "none" else None
        dW = torch.zeros_like(W) if case["grads"] == "both" else None
        for a in range(0, N, 512):       # rows in pieces: the logits of 512 rows at a time
            z = torch.matmul(x[a:a + 512], W.mT)
            y = s["y"][a:a + 512].long()
            keep = (y != -1).nonzero()[:, 0]
            z, y = z[keep], y[keep]
            lse = torch.logsumexp(z, 1)
            row_loss[a + keep] = lse - z[torch.arange(len(y), device="cuda"), y]
            if dx is not None:
                p = torch.exp(z - lse[:, None])
                p[torch.arange(len(y), device="cuda"), y] -= 1.0
                p *= s["S"] / N
                dx[a + keep] = torch.matmul(p, W)
                if dW is not None:
                    dW.addmm_(p.mT, x[a + keep])
            del z
        out = {"row_loss": row_loss, "loss": row_loss.mean()}
        if dx is not None:
            out["dx"] = dx
        if dW is not None:
            out["dW"] = dW
        return out
    B, tau = case["B"], case["tau"]
    dz = torch.empty(B, case["C"], dtype=torch.float64, device="cuda")
    row_loss = torch.zeros(B, dtype=torch.float64, device="cuda")
    for a in range(0, B, 256):
        logp = torch.log_softmax(s["z"][a:a + 256].double() / tau, 1)
        idx = s["idx"][a:a + 256].long()
        has = (idx >= 0).any(1)
        q = torch.softmax((s["t"][a:a + 256].double() / tau).masked_fill(idx < 0, -math.inf), 1).nan_to_num(0.0)
        kl = torch.xlogy(q, q) - q * logp.gather(1, idx.clamp(min=0))
        row_loss[a:a + 256] = kl.sum(1) * tau ** 2
        p = logp.exp() * has[:, None]
        p.scatter_add_(1, idx.clamp(min=0), -q)
        dz[a:a + 256] = p * tau * s["S"] / B
    return {"dz": dz, "row_loss": row_loss, "loss": row_loss.mean()}


def work(case):
    if case["op"] == "ln_fwd":
        n = case["rows"] * case["cols"]      # x in, y out; the scale and shift vectors; two statistics a row
        return {"bytes": 4 * n + 2 * case["cols"] * (2 if case["beta"] else 1) + 8 * case["rows"], "flops": 8 * n}
    if case["op"] == "ln_bwd":
        n = case["rows"] * case["cols"]      # dy and x in, dx out; gamma, dgamma (and dbeta); two statistics a row
        return {"bytes": 6 * n + 2 * case["cols"] * (3 if case["beta"] else 2) + 8 * case["rows"], "flops": 14 * n}
    if case["op"] == "lce":
        N, V, H = case["N"], case["V"], case["H"]
        products = {"none": 1, "dx": 2, "both": 3}[case["grads"]]
        moved = 2 * N * H + 2 * V * H + 8 * N + 4 + (2 * N * H if products > 1 else 0) + (2 * V * H if products > 2 else 0)
        return {"bytes": moved, "flops": 2 * products * N * V * H}
    B, C, K = case["B"], case["C"], case["K"]      # logits in, gradient out; the teacher's values and classes; a loss a row
    return {"bytes": 4 * B * C + 6 * B * K + 4 * B + 4, "flops": 8 * B * C}
