"""Cases for measuring the operators around the quantized layers of a transformer's training step: layer norm, the
8-bit activation checkpoints (with the GELU and the layer norm that use them) and the language-model loss.

`run` computes an operator either in plain torch operations in 32 bits (`own = False`) or through the library
(`own = True`).  `exact` is the same operator written from its definition in 64 bits.
"""
import math

import torch

own = False

EPS = 1e-5
GROUP = 128          # elements of a row that share a checkpoint scale
TINY = 2.0 ** -100   # groups whose largest magnitude is below this are stored as zeros

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # layer norm ---------------------------------------------------------------------------------
        # one token of a 768-wide encoder, forward only: pure latency
        {"name": "ln_fwd_one_token", "op": "ln_fwd", "rows": 1, "cols": 768, "dtype": "bf16"},
        # fp32 activations, a width that is no multiple of a warp's vectors, a prime number of rows
        {"name": "ln_step_odd_f32", "op": "ln_step", "rows": 1021, "cols": 1000, "dtype": "f32"},
        # the norm of a 24-layer, 1024-wide encoder at batch 24 x 384 tokens
        {"name": "ln_step_9216x1024", "op": "ln_step", "rows": 9216, "cols": 1024, "dtype": "bf16"},
        # a wide model on a long batch: 128 MiB per tensor, nothing fits the cache
        {"name": "ln_step_16384x4096", "op": "ln_step", "rows": 16384, "cols": 4096, "dtype": "bf16"},
        # 8-bit activation checkpoints ---------------------------------------------------------------
        # store and load of an fp32 tensor with a ragged last group and an odd number of rows
        {"name": "ckpt_roundtrip_odd_f32", "op": "ckpt", "rows": 4093, "cols": 1040, "dtype": "f32"},
        # the activation of a few tokens: latency of the two calls
        {"name": "ckpt_gelu_few_tokens", "op": "gelu_step", "rows": 61, "cols": 1504, "dtype": "bf16"},
        # the feed-forward activation of the 1024-wide encoder (4096 hidden channels)
        {"name": "ckpt_gelu_9216x4096", "op": "gelu_step", "rows": 9216, "cols": 4096, "dtype": "bf16"},
        # the same encoder's norm, with its input kept in 8 bits between forward and backward
        {"name": "ckpt_ln_9216x1024", "op": "ln_ckpt_step", "rows": 9216, "cols": 1024, "dtype": "bf16"},
        # language-model loss ------------------------------------------------------------------------
        # scoring one token: the vocabulary's matrix is read once, nothing else counts
        {"name": "lm_fwd_one_token", "op": "lm_fwd", "tokens": 1, "vocab": 32000, "dim": 1024, "dtype": "bf16"},
        # evaluation of a batch on a 768-wide model with an odd vocabulary
        {"name": "lm_fwd_2048x49999", "op": "lm_fwd", "tokens": 2048, "vocab": 49999, "dim": 768, "dtype": "bf16"},
        # one ragged micro-batch of a training step, a width that is no multiple of 64
        {"name": "lm_step_509x30521", "op": "lm_step", "tokens": 509, "vocab": 30521, "dim": 1000, "dtype": "bf16"},
        # the training step of a large vocabulary: 4 GB of fp32 logits if they were kept
        {"name": "lm_step_8192x128000", "op": "lm_step", "tokens": 8192, "vocab": 128000, "dim": 2048, "dtype": "bf16"},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["ln_fwd", "ln_step", "ckpt", "gelu_step", "ln_ckpt_step", "lm_fwd", "lm_step", "lm_step"])
    if op.startswith("lm"):
        while True:
            t, v, d = _log_int(rng, 1, 8192), _log_int(rng, 1000, 128000), 8 * _log_int(rng, 32, 256)
            if t * v * d <= 8192 * 128000 * 2048:
                return {"op": op, "tokens": t, "vocab": v, "dim": d, "dtype": "bf16"}
    unit = 8 if op.startswith("ln_") and op != "ln_ckpt_step" else 16
    while True:
        rows, cols = _log_int(rng, 1, 16384), unit * _log_int(rng, 64 // unit, 8192 // unit)
        if rows * cols <= 16384 * 4096:
            return {"op": op, "rows": rows, "cols": cols, "dtype": rng.choice(["bf16", "bf16", "f32"])}


def work(case):
    op = case["op"]
    if op.startswith("lm"):
        t, v, d = case["tokens"], case["vocab"], case["dim"]
        mats = 2 * (t * d + v * d)
        if op == "lm_fwd":
            return {"bytes": mats + 12 * t, "flops": 2 * t * v * d}
        # the three products of the step; that the logits are formed twice is the price of not keeping them
        return {"bytes": 2 * mats + 16 * t, "flops": 6 * t * v * d}
    n, rows, cols, e = case["rows"] * case["cols"], case["rows"], case["cols"], SIZE[case["dtype"]]
    kept = n + 4 * rows * -(-cols // GROUP)      # a checkpoint's codes and scales
    if op == "ln_fwd":
        return {"bytes": 2 * e * n + 8 * rows + 8 * cols, "flops": 8 * n}
    if op == "ln_step":
        return {"bytes": 5 * e * n + 16 * rows + 20 * cols, "flops": 20 * n}
    if op == "ln_ckpt_step":
        return {"bytes": 4 * e * n + 2 * kept + 16 * rows + 20 * cols, "flops": 24 * n}
    if op == "ckpt":
        return {"bytes": 2 * e * n + 2 * kept, "flops": 6 * n}
    return {"bytes": 4 * e * n + 2 * kept, "flops": 40 * n}                  # gelu_step


# ------------------------------------------------------------------------------------------------ inputs
def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 1000003 + 17)
    dt = DTYPES[case["dtype"]]

    def normal(*shape, std=1.0, mean=0.0, dtype=torch.float32):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).mul_(std).add_(mean).to(dtype)

    s = dict(case)
    if case["op"].startswith("lm"):
        t, v, d = case["tokens"], case["vocab"], case["dim"]
        # hidden states as a final layer norm leaves them; logits with a standard deviation of about 3
        s["H"] = normal(t, d, dtype=dt)
        s["W"] = normal(v, d, std=3.0 / math.sqrt(d), dtype=dt)
        labels = torch.randint(0, v, (t,), generator=g, device="cuda", dtype=torch.int32)
        skip = torch.rand((t,), generator=g, device="cuda") < 0.1      # padding: no target
        s["labels"] = torch.where(skip, torch.full_like(labels, -1), labels)
        valid = (s["labels"] >= 0)
        s["dloss"] = valid.float() / valid.sum().clamp(min=1).float()  # gradient of the mean over the targets
        return s
    m, c = case["rows"], case["cols"]
    # a residual stream: per-channel spread, a few channels several times larger, rows off zero
    spread = torch.exp(normal(c, std=0.5))
    spread = torch.where(torch.rand((c,), generator=g, device="cuda") < 0.01, spread * 8, spread)
    s["x"] = (normal(m, c) * spread + normal(m, 1, std=0.3, mean=0.3)).to(dt)
    if case["op"] in ("gelu_step", "ln_step", "ln_ckpt_step"):
        s["dy"] = normal(m, c, dtype=dt)
    if case["op"].startswith("ln"):
        s["gamma"], s["beta"] = normal(c, std=0.2, mean=1.0), normal(c, std=0.2)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        from paper_2411_11038_b200 import binding as B
        ctx = B.Context(0)
        if case["op"].startswith("lm"):
            s["plan"] = B.LmLossPlan(ctx, case["tokens"], case["vocab"], case["dim"], "cuda",
                                     backward=case["op"] == "lm_step")
        else:
            m, c, dt = case["rows"], case["cols"], DTYPES[case["dtype"]]
            if case["op"].startswith("ln"):
                s["plan"] = B.LayerNormPlan(ctx, m, c, dt, "cuda", eps=EPS, backward=case["op"] != "ln_fwd")
            elif case["op"] == "gelu_step":
                s["plan"] = B.GeluPlan(ctx, m, c, dt, "cuda")
            if case["op"] in ("ckpt", "gelu_step", "ln_ckpt_step"):
                s["ckpt"] = B.Checkpoint(ctx, m, c, "cuda")
            if case["op"] == "ckpt":
                s["back"] = torch.empty_like(s["x"])
    return s


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    op = s["op"]
    if op == "ln_fwd":
        y = s["plan"].fwd(s["x"], s["gamma"], s["beta"])
        return {"y": y, "mean": s["plan"].mean, "rstd": s["plan"].rstd}
    if op == "ln_step":
        y = s["plan"].fwd(s["x"], s["gamma"], s["beta"])
        return {"y": y, **s["plan"].bwd(s["dy"], s["gamma"], x=s["x"])}
    if op == "ln_ckpt_step":
        y = s["plan"].fwd(s["x"], s["gamma"], s["beta"], save=s["ckpt"])
        return {"y": y, **s["plan"].bwd(s["dy"], s["gamma"], saved=s["ckpt"])}
    if op == "ckpt":
        s["ckpt"].store(s["x"])
        return {"x": s["ckpt"].load(out=s["back"])}
    if op == "gelu_step":
        y = s["plan"].fwd(s["x"], save=s["ckpt"])
        return {"y": y, "dx": s["plan"].bwd(s["dy"], saved=s["ckpt"])}
    loss = s["plan"].fwd(s["H"], s["W"], s["labels"])
    if op == "lm_fwd":
        return {"loss": loss, "lse": s["plan"].lse}
    return {"loss": loss, **s["plan"].bwd(s["H"], s["W"], s["labels"], s["dloss"])}


def _through_8_bits(x):
    """x after a checkpoint: groups of a row in 8-bit codes of one scale each."""
    m, c = x.shape
    pad = -c % GROUP
    g = torch.nn.functional.pad(x, (0, pad)).view(m, -1, GROUP)
    top = g.abs().amax(dim=2, keepdim=True)
    full = torch.full_like(top, 127.0)
    live = top >= TINY
    scale = torch.where(live, torch.div(top, full), torch.zeros_like(top))
    factor = torch.where(live, torch.div(full, top), torch.zeros_like(top))
    return (torch.round(g * factor) * scale).view(m, -1)[:, :c]


def _ln_backward(dy, x, gamma, mean, rstd):
    xh = (x - mean) * rstd
    g = dy * gamma
    dx = rstd * (g - g.mean(dim=1, keepdim=True) - xh * (g * xh).mean(dim=1, keepdim=True))
    return dx, (dy * xh).sum(dim=0), dy.sum(dim=0)


def _run_plain(s):
    op = s["op"]
    if op.startswith("lm"):
        h, w, labels = s["H"].float(), s["W"].float(), s["labels"].long()
        valid = labels >= 0
        at = labels.clamp(min=0)[:, None]
        logits = h @ w.t()
        top = logits.amax(dim=1, keepdim=True)
        lse = top[:, 0] + torch.log(torch.exp(logits - top).sum(dim=1))
        loss = torch.where(valid, lse - logits.gather(1, at)[:, 0], torch.zeros_like(lse))
        if op == "lm_fwd":
            return {"loss": loss, "lse": lse}
        scale = torch.where(valid, s["dloss"], torch.zeros_like(lse))[:, None]
        g = torch.exp(logits - lse[:, None]) * scale
        g.scatter_add_(1, at, -scale)
        return {"loss": loss, "dH": (g @ w).to(s["H"].dtype), "dW": (g.t() @ h).to(s["W"].dtype)}
    dt, x = s["x"].dtype, s["x"].float()
    if op == "ckpt":
        return {"x": _through_8_bits(x).to(dt)}
    if op == "gelu_step":
        y = x * (0.5 * (1.0 + torch.erf(x * math.sqrt(0.5))))
        x = _through_8_bits(x)
        slope = 0.5 * (1.0 + torch.erf(x * math.sqrt(0.5))) + x * torch.exp(x * x * -0.5) * (1.0 / math.sqrt(2.0 * math.pi))
        return {"y": y.to(dt), "dx": (s["dy"].float() * slope).to(dt)}
    mean = x.mean(dim=1, keepdim=True)
    mid = x - mean
    rstd = torch.rsqrt((mid * mid).mean(dim=1, keepdim=True) + EPS)
    y = (mid * rstd * s["gamma"] + s["beta"]).to(dt)
    if op == "ln_fwd":
        return {"y": y, "mean": mean[:, 0], "rstd": rstd[:, 0]}
    if op == "ln_ckpt_step":
        x = _through_8_bits(x)
    dx, dgamma, dbeta = _ln_backward(s["dy"].float(), x, s["gamma"], mean, rstd)
    return {"y": y, "dx": dx.to(dt), "dgamma": dgamma, "dbeta": dbeta}


# ------------------------------------------------------------------------------------------------ in 64 bits
def _kept_64(x):
    """What a checkpoint of x stands for: the code of an element is the nearest integer (ties to even) to
    fl32(x * fl32(127 / a)), its value the code times fl32(a / 127), with a the largest magnitude of its group."""
    out = torch.empty_like(x)
    for c0 in range(0, x.shape[1], GROUP):
        part = x[:, c0:c0 + GROUP]
        a = part.abs().max(dim=1, keepdim=True).values
        zero = a < TINY
        a = torch.where(zero, torch.ones_like(a), a)
        unit, per = (a / 127.0).float().double(), (127.0 / a).float().double()
        code = torch.round((part * per).float().double())
        out[:, c0:c0 + GROUP] = torch.where(zero, torch.zeros_like(code), (code * unit).float().double())
    return out


def exact(case, seed):
    s = _inputs(case, seed)
    op = case["op"]
    if op.startswith("lm"):
        h, w, labels = s["H"].double(), s["W"].double(), s["labels"].long()
        t, v = h.shape[0], w.shape[0]
        loss, norm = torch.zeros(t, dtype=torch.float64, device="cuda"), torch.zeros(t, dtype=torch.float64, device="cuda")
        dh, dw = torch.zeros_like(h), torch.zeros_like(w)
        for t0 in range(0, t, 1024):
            rows = slice(t0, min(t, t0 + 1024))
            z = h[rows] @ w.t()
            norm[rows] = torch.logsumexp(z, dim=1)
            hit = torch.nonzero(labels[rows] >= 0)[:, 0]
            loss[rows][hit] = norm[rows][hit] - z[hit, labels[rows][hit]]
            if op == "lm_step":
                z = torch.softmax(z, dim=1)
                z[hit, labels[rows][hit]] -= 1.0
                z *= torch.where(labels[rows] >= 0, s["dloss"][rows].double(), torch.zeros((), dtype=torch.float64, device="cuda"))[:, None]
                dh[rows] = z @ w
                dw += z.t() @ h[rows]
        return {"loss": loss, "lse": norm} if op == "lm_fwd" else {"loss": loss, "dH": dh, "dW": dw}
    x = s["x"].double()
    if op == "ckpt":
        return {"x": _kept_64(x)}
    if op == "gelu_step":
        kept = _kept_64(x)
        slope = torch.special.ndtr(kept) + kept * torch.exp(-kept * kept / 2) / math.sqrt(2 * math.pi)
        return {"y": x * torch.special.ndtr(x), "dx": s["dy"].double() * slope}
    gamma, beta = s["gamma"].double(), s["beta"].double()
    var, mean = torch.var_mean(x, dim=1, unbiased=False, keepdim=True)
    rstd = (var + EPS) ** -0.5
    y = (x - mean) * rstd * gamma + beta
    if op == "ln_fwd":
        return {"y": y, "mean": mean[:, 0], "rstd": rstd[:, 0]}
    n, dy = x.shape[1], s["dy"].double()
    hat = ((_kept_64(x) if op == "ln_ckpt_step" else x) - mean) * rstd
    inner = torch.stack([(dy @ gamma) / n, ((dy * hat) @ gamma) / n])
    dx = rstd * (dy * gamma - inner[0][:, None] - hat * inner[1][:, None])
    return {"y": y, "dx": dx, "dgamma": torch.einsum("mc,mc->c", dy, hat), "dbeta": torch.einsum("mc->c", dy)}
