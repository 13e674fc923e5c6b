"""The two ends of a language model's backward pass, as cases that can be timed.

  score   softmax cross entropy of the last layer's logits X . W^T against one target per token, the logits never kept:
          the loss and the log of the softmax's denominator, per token
  loss    the same and its gradient: the loss-scaled error of the hidden states and the weights' gradient, as halves or as
          8-bit codes
  ortho   a momentum step whose direction is orthogonalised by Newton-Schulz products before it is applied to the
          half-precision master weights

M tokens, N classes (the vocabulary), K features; a matrix of weights is [rows, cols].  Without `own` every operator is
computed in its plain form, with it by the framework's entry points.
"""
import math

import torch

own = False

SEED = 0x1905_1233_4000_0000
QUINTIC = (3.4445, -4.7750, 2.0315)  # coefficients of a Newton-Schulz step on the singular values
STEPS, MOMENTUM, DECAY = 5, 0.95, 0.01
LARGEST_LOSS, LARGEST_ORTHO = 8192 * 131072 * 2048, 4096 * 4096 * 8192


def listed():
    return [
        # the log-probability of one next token: latency, then the weights' bytes
        {"name": "score 1 token", "kind": "score", "M": 1, "N": 32000, "K": 512, "ignored": 0.0, "x8": False},
        # ranking a text by its likelihood; hidden states as the 8-bit layers leave them, no size a round number
        {"name": "score 1021 tokens", "kind": "score", "M": 1021, "N": 32003, "K": 1000, "ignored": 0.1, "x8": True},
        # the classifier of an image network on one batch
        {"name": "loss 1000 classes", "kind": "loss", "M": 256, "N": 1000, "K": 2048, "ignored": 0.0, "x8": False,
         "weighted": False, "codes": False, "sr": False},
        # a base translation network, sentences padded to one length, a weight per token
        {"name": "loss 4096 tokens", "kind": "loss", "M": 4096, "N": 32000, "K": 512, "ignored": 0.2, "x8": False,
         "weighted": True, "codes": False, "sr": False},
        # sentences as they come, everything that leaves the layer in 8 bits and stochastically rounded
        {"name": "loss 6007 tokens", "kind": "loss", "M": 6007, "N": 37003, "K": 1000, "ignored": 0.0, "x8": True,
         "weighted": False, "codes": True, "sr": True},
        # a large vocabulary: the matrix cores decide
        {"name": "loss 8192 tokens", "kind": "loss", "M": 8192, "N": 131072, "K": 2048, "ignored": 0.0, "x8": False,
         "weighted": False, "codes": False, "sr": False},
        # the smallest layer: launches decide
        {"name": "ortho 256x256", "kind": "ortho", "batch": 1, "rows": 256, "cols": 256, "sr": True, "w8": True},
        # a lowered convolution's weights: tall and narrow
        {"name": "ortho 1152x128", "kind": "ortho", "batch": 1, "rows": 1152, "cols": 128, "sr": True, "w8": False},
        # the projections of all attention blocks of a base translation network in one call
        {"name": "ortho 24x512x512", "kind": "ortho", "batch": 24, "rows": 512, "cols": 512, "sr": True, "w8": True},
        # feed-forward layer of a big translation network
        {"name": "ortho 1024x4096", "kind": "ortho", "batch": 1, "rows": 1024, "cols": 4096, "sr": True, "w8": True},
        # no size a multiple of anything, rounded to nearest
        {"name": "ortho 2001x1013", "kind": "ortho", "batch": 1, "rows": 2001, "cols": 1013, "sr": False, "w8": True},
        # feed-forward layer of a large network: the matrix cores decide
        {"name": "ortho 4096x8192", "kind": "ortho", "batch": 1, "rows": 4096, "cols": 8192, "sr": True, "w8": True},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A layer's width: mostly a multiple of 64, now and then of 8 or of nothing."""
    unit = rng.choices([64, 8, 1], [6, 2, 2])[0]
    return max(unit, (_log_int(rng, lo, hi) + unit // 2) // unit * unit)


def draw(rng):
    kind = rng.choice(["score", "loss", "loss", "ortho", "ortho"])
    if kind == "ortho":
        while True:
            batch, rows, cols = rng.choice([1, 1, 1, 2, 6, 24]), _width(rng, 16, 8192), _width(rng, 16, 8192)
            if batch * rows * cols * min(rows, cols) <= LARGEST_ORTHO:
                return {"kind": kind, "batch": batch, "rows": rows, "cols": cols, "sr": rng.random() < 0.7, "w8": rng.random() < 0.7}
    while True:
        M, N, K = _log_int(rng, 1, 16384), _width(rng, 16, 131072), _width(rng, 32, 4096)
        if M * N * K <= LARGEST_LOSS // 2:
            break
    c = {"kind": kind, "M": M, "N": N, "K": K, "ignored": rng.choice([0.0, 0.0, 0.1, 0.3]), "x8": rng.random() < 0.3}
    if kind == "loss":
        codes = rng.random() < 0.4
        c |= {"weighted": rng.random() < 0.3, "codes": codes, "sr": codes and rng.random() < 0.6}
    return c


# ---------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------
def _tokens(c, seed):
    """Hidden states whose logits are about N(0, 1), but for the target's, which stands out by 0 .. 2 ln N as it does in a
    model that has learnt something; targets as frequent as words are; the last tokens without a target (-100) are padding."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    M, N, K = c["M"], c["N"], c["K"]
    s = {"case": c}
    s["w"] = torch.randn((N, K), generator=gen, device="cuda").mul_(K ** -0.5).half()
    u = torch.rand((M, 2), generator=gen, device="cuda", dtype=torch.float64)
    t = (N ** u[:, 0]).long().sub_(1).clamp_(0, N - 1)
    x = torch.randn((M, K), generator=gen, device="cuda")
    x += (2 * math.log(N + 1) * u[:, 1:]).float() * s["w"][t].float()
    s["x"] = x.to(torch.float8_e5m2).view(torch.uint8) if c["x8"] else x.half()
    n_ignored = int(c["ignored"] * M)
    if n_ignored:
        t[M - n_ignored:] = -100
    s["targets"] = t
    s["scale"] = 2.0 ** 14 / max(1, M - n_ignored)  # loss scale over the number of tokens
    s["dloss"] = torch.rand(M, generator=gen, device="cuda") * 1.5 + 0.25 if c.get("weighted") else None
    return s


def _weights(c, seed):
    """Master weights, the momentum so far, and gradient codes: a few strong directions and noise, as gradients have."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    b, r, k = shape = (c["batch"], c["rows"], c["cols"])

    def gradient():
        rank = max(1, min(r, k) // 16)
        strong = torch.randn((b, r, rank), generator=gen, device="cuda") @ torch.randn((b, rank, k), generator=gen, device="cuda")
        return strong.mul_(0.5 * rank ** -0.5).add_(torch.randn(shape, generator=gen, device="cuda"))
    s = {"case": c, "inv_loss_scale": 2.0 ** -14}
    s["w16"] = (torch.rand(shape, generator=gen, device="cuda") * 2 - 1).mul_(math.sqrt(6.0 / (r + k))).half()
    s["velocity"] = gradient().mul_(5e-5)
    s["g8"] = gradient().mul_(0.16).to(torch.float8_e5m2).view(torch.uint8)
    s["lr"] = 0.02 * 0.2 * math.sqrt(max(r, k))  # a step as long as ADAM's
    return s


def prepare(case, seed):
    return _weights(case, seed) if case["kind"] == "ortho" else _tokens(case, seed)


# ---------------------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------------------
def _random16(n, offset):
    """16 bits per element: Philox4x32-10 (key SEED), block i / 8, halfword i % 8."""
    mask = 0xFFFFFFFF
    blk = torch.arange((n + 7) // 8, device="cuda", dtype=torch.int64)
    c = [blk & mask, blk >> 32, torch.full_like(blk, offset & mask), torch.full_like(blk, offset >> 32)]
    ka, kb = SEED & mask, SEED >> 32
    for _ in range(10):
        p0, p1 = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [((p1 >> 32) & mask) ^ c[1] ^ ka, p1 & mask, ((p0 >> 32) & mask) ^ c[3] ^ kb, p0 & mask]
        ka, kb = (ka + 0x9E3779B9) & mask, (kb + 0xBB67AE85) & mask
    words = torch.stack(c, 1).reshape(-1)
    return torch.stack([words & 0xFFFF, words >> 16], 1).reshape(-1)[:n]


def _stochastic(x, drop, offset):
    """Finite FP32 values to the format with exponents of 5 bits that drops `drop` bits of FP32's fraction, as codes:
    the magnitude goes up by one where the upper 16 bits of what is dropped and 16 random bits carry."""
    flat = x.reshape(-1)
    r = _random16(flat.numel(), offset)
    bits = flat.view(torch.int32).long()
    a = bits & 0x7FFFFFFF
    t = a - 0x38000000
    dropped = t & ((1 << drop) - 1)
    dropped = dropped >> (drop - 16) if drop >= 16 else dropped << (16 - drop)
    normal = (t >> drop) + ((dropped + r) >> 16)
    quanta = (flat.abs().double() * 2.0 ** (53 - drop)).long()  # below the smallest normal: units of 2^-16 of a quantum
    low = (quanta + r) >> 16
    code = torch.where(a >= 0x38800000, normal, low).clamp(max=0x7C00 >> (drop - 13))
    width = 29 - drop
    return (code | ((bits >> 31) & 1) << (width - 1)).reshape(x.shape)


def _half(x, sr, offset):
    return _stochastic(x, 13, offset).to(torch.int16).view(torch.float16) if sr else x.half()


def _eight(x, sr, offset):
    return _stochastic(x, 21, offset).to(torch.uint8).view(torch.float8_e5m2) if sr else x.to(torch.float8_e5m2)


def _plain_cross_entropy(s):
    c = s["case"]
    x = s["x"].view(torch.float8_e5m2).float() if c["x8"] else s["x"].float()
    w = s["w"].float()
    z = x @ w.t()
    given = s["targets"] >= 0
    at = s["targets"].clamp(min=0)[:, None]
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    lse = (top + torch.log(total))[:, 0]
    # -log p of the target as log(1 + what the others have beside it): near zero lse - z loses every digit
    others = e.scatter(1, at, 0.0).sum(1)
    over = top[:, 0] - z.gather(1, at)[:, 0]
    loss = torch.where(over < 64, torch.log1p(others * torch.exp(over)), over + torch.log(others))
    loss = torch.where(given, loss, 0.0)
    if c["kind"] == "score":
        return {"loss": loss, "lse": lse}
    del z
    e /= total
    e.scatter_add_(1, at, torch.full_like(lse, -1.0)[:, None])
    per_token = s["scale"] * (s["dloss"] if s["dloss"] is not None else torch.ones_like(lse))
    e *= per_token[:, None]
    e[~given] = 0.0
    dx, dw = e @ w, e.t() @ x
    if c["codes"]:
        return {"loss": loss, "lse": lse, "dx": _eight(dx, c["sr"], 1), "dw": _eight(dw, c["sr"], 2)}
    return {"loss": loss, "lse": lse, "dx": dx.half(), "dw": dw.half()}


def _plain_ortho(s):
    c = s["case"]
    g = s["g8"].view(torch.float8_e5m2).float() * s["inv_loss_scale"]
    s["velocity"].mul_(MOMENTUM).add_(g)
    o = g + MOMENTUM * s["velocity"]
    tall = c["rows"] > c["cols"]
    o = o.transpose(1, 2).contiguous() if tall else o
    norm = o.double().square().sum((1, 2), keepdim=True).sqrt()
    o = torch.where(norm > 0, o / norm, 0.0).float()
    c1, c3, c5 = QUINTIC
    for _ in range(STEPS):
        a = o @ o.transpose(1, 2).contiguous()
        o = c1 * o + (c3 * a + c5 * (a @ a)) @ o
    o = o.transpose(1, 2).contiguous() if tall else o
    w = s["w16"].float()
    s["w16"].copy_(_half(w - s["lr"] * (o + DECAY * w), c["sr"], 3))
    out = {"w16": s["w16"], "velocity": s["velocity"]}
    if c["w8"]:
        out["w8"] = s["w16"].to(torch.float8_e5m2)
    return out


# ---------------------------------------------------------------------------------------
# the framework's entry points
# ---------------------------------------------------------------------------------------
def _empty(dtype, *shape):
    return torch.empty(shape, dtype=dtype, device="cuda")


def _own_cross_entropy(s):
    import paper_1905_12334_amd as mp8
    c = s["case"]
    M, N, K = c["M"], c["N"], c["K"]
    if "out" not in s:  # what a program allocates once
        out = s["out"] = {"loss": _empty(torch.float32, M), "lse": _empty(torch.float32, M)}
        need = mp8.softmax_xent_fwd_workspace_bytes(M, N, K)
        if c["kind"] == "loss":
            dtype = torch.uint8 if c["codes"] else torch.float16
            out |= {"dx": _empty(dtype, M, K), "dw": _empty(dtype, N, K)}
            need = max(need, mp8.softmax_xent_bwd_workspace_bytes(M, N, K))
        s["workspace"] = _empty(torch.uint8, max(need, 16))
    out, ws = s["out"], s["workspace"]
    mp8.softmax_xent_fwd_fp16(M, N, K, s["x"], s["w"], s["targets"], out["loss"], out["lse"], workspace=ws)
    if c["kind"] == "score":
        return out
    if c["codes"]:
        mp8.softmax_xent_bwd_fp16(M, N, K, s["x"], s["w"], s["targets"], out["loss"], out["lse"], dx8=out["dx"], dw8=out["dw"], dloss=s["dloss"],
                                  scale=s["scale"], round=mp8.SR if c["sr"] else mp8.RNE, seed=SEED, dx_offset=1, dw_offset=2,
                                  workspace=ws)
        return {k: v.view(torch.float8_e5m2) if v.dtype == torch.uint8 else v for k, v in out.items()}
    mp8.softmax_xent_bwd_fp16(M, N, K, s["x"], s["w"], s["targets"], out["loss"], out["lse"], dx16=out["dx"], dw16=out["dw"], dloss=s["dloss"],
                              scale=s["scale"], workspace=ws)
    return out


def _own_ortho(s):
    import paper_1905_12334_amd as mp8
    c = s["case"]
    if "workspace" not in s:
        s["workspace"] = _empty(torch.uint8, max(16, mp8.orthogonal_momentum_workspace_bytes(c["batch"], c["rows"], c["cols"])))
        s["w8"] = _empty(torch.uint8, *s["w16"].shape) if c["w8"] else None
    mp8.orthogonal_momentum_fp16_sr(s["w16"], s["velocity"], s["g8"], s["lr"], s["inv_loss_scale"], MOMENTUM, nesterov=True,
                                    weight_decay=DECAY, steps=STEPS, round=mp8.SR if c["sr"] else mp8.RNE, seed=SEED, offset=3,
                                    w8_out=s["w8"], workspace=s["workspace"])
    out = {"w16": s["w16"], "velocity": s["velocity"]}
    if c["w8"]:
        out["w8"] = s["w8"].view(torch.float8_e5m2)
    return out


def run(state):
    if state["case"]["kind"] == "ortho":
        return _own_ortho(state) if own else _plain_ortho(state)
    return _own_cross_entropy(state) if own else _plain_cross_entropy(state)


# ---------------------------------------------------------------------------------------
# in 64 bits, from the definitions
# ---------------------------------------------------------------------------------------
def _exact_cross_entropy(c, s):
    """A block of tokens at a time; results are not rounded, so that 8-bit gradients have none here."""
    x = (s["x"].view(torch.float8_e5m2) if c["x8"] else s["x"]).double()
    w = s["w"].double()
    M, N = c["M"], c["N"]
    loss, lse = torch.zeros(M, dtype=torch.float64, device="cuda"), torch.zeros(M, dtype=torch.float64, device="cuda")
    dx, dw = torch.zeros_like(x), torch.zeros_like(w)
    step = max(1, 2 ** 28 // N)
    for i in range(0, M, step):
        rows = slice(i, min(M, i + step))
        z = x[rows] @ w.t()
        lse[rows] = torch.logsumexp(z, 1)
        t = s["targets"][rows]
        live = torch.nonzero(t >= 0)[:, 0]
        behind = z - z[torch.arange(len(t)), t.clamp(min=0)][:, None]
        behind[live, t[live]] = -math.inf
        loss[rows.start + live] = torch.nn.functional.softplus(torch.logsumexp(behind, 1), threshold=100)[live]
        if c["kind"] == "score":
            continue
        p = torch.exp(z - lse[rows][:, None])
        p[live, t[live]] -= 1
        factor = torch.zeros(len(t), dtype=torch.float64, device="cuda")
        factor[live] = s["scale"] * (s["dloss"][rows][live].double() if s["dloss"] is not None else 1.0)
        p *= factor[:, None]
        dx[rows] = p @ w
        dw += p.t() @ x[rows]
    if c["kind"] == "score":
        return {"loss": loss, "lse": lse}
    return {"loss": loss, "lse": lse, "dx": None if c["codes"] else dx, "dw": None if c["codes"] else dw}


def _exact_ortho(c, s):
    """Matrix by matrix; the polynomial from its odd powers; the new weights before they are rounded to half (their 8-bit
    copies are what that rounding makes of them, and have no value here)."""
    w, v, g = s["w16"].double(), s["velocity"].double(), s["g8"].view(torch.float8_e5m2).double() * s["inv_loss_scale"]
    v = MOMENTUM * v + g
    u = MOMENTUM * v + g
    for i in range(c["batch"]):
        y = u[i] / torch.linalg.norm(u[i])
        if c["rows"] < c["cols"]:
            y = y.t().contiguous()
        for _ in range(STEPS):
            gram = y.t() @ y
            cubed = y @ gram
            y = QUINTIC[0] * y + QUINTIC[1] * cubed + QUINTIC[2] * (cubed @ gram)
        u[i] = y.t() if c["rows"] < c["cols"] else y
    w = (1.0 - s["lr"] * DECAY) * w - s["lr"] * u
    return {"w16": w, "velocity": v, "w8": None}


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_ortho(case, s) if case["kind"] == "ortho" else _exact_cross_entropy(case, s)


# ---------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------
def work(case):
    c = case
    if c["kind"] == "ortho":
        # codes and momentum in, momentum and weights out; per step a symmetric Gram matrix, its symmetric square and one
        # more product
        b, m, n = c["batch"], min(c["rows"], c["cols"]), max(c["rows"], c["cols"])
        return {"bytes": b * m * n * (1 + 8 + 4 + (1 if c["w8"] else 0)), "flops": STEPS * b * (3 * m * m * n + m ** 3)}
    M, N, K = c["M"], c["N"], c["K"]
    x = 1 if c["x8"] else 2
    if c["kind"] == "score":
        return {"bytes": x * M * K + 2 * N * K + 16 * M, "flops": 2 * M * N * K}
    out = 1 if c["codes"] else 2
    return {"bytes": (x + out) * M * K + (2 + out) * N * K + (20 if c["weighted"] else 16) * M, "flops": 6 * M * N * K}
