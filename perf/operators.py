"""The cases on which three operators of the library are measured, with their plain forms.

  cross entropy   token cross-entropy of an LM head over a large vocabulary, with the gradients of the
                  hidden states and of the head, without the [T, V] logits in memory
  norm            the join of a block's branch with the residual stream: norm of the branch, gate, scaled
                  residual, and the norm that the next block (or the LM head) reads; both directions
  linear          x W^T with bias, activation and residual in the epilogue; both directions

`run` with `own` false is the plain form, elementary torch operations in 32 bits; with `own` true it makes
the calls a user makes of this repository's package.
"""

import math

import numpy as np
import torch

own = False

DEV = "cuda"
IGNORE = -100
SEG = 512            # packed segments of the cross-entropy cases
PROMPT = 153         # their leading tokens without loss (30 %)
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")


# ------------------------------------------------------------------------------------------------
# cases
# ------------------------------------------------------------------------------------------------
def listed():
    return [
        # the log-probability of one sampled token under the ~1B student's head
        {"name": "ce_score_token", "op": "ce", "T": 1, "d": 1536, "V": 151936, "tau": 1.0, "step": False,
         "masked": False, "weighted": False},
        # the smallest step, where the launches are what counts
        {"name": "ce_step_tiny", "op": "ce", "T": 256, "d": 64, "V": 1000, "tau": 1.0, "step": True,
         "masked": True, "weighted": False},
        # one odd row of a batch: a vocabulary that fills no tile, token weights, a temperature
        {"name": "ce_step_ragged", "op": "ce", "T": 2047, "d": 2048, "V": 32003, "tau": 2.0, "step": True,
         "masked": True, "weighted": True},
        # supervised step of the ~1B student on one packed row, 30 % prompt tokens
        {"name": "ce_step_1b", "op": "ce", "T": 8192, "d": 1536, "V": 151936, "tau": 1.0, "step": True,
         "masked": True, "weighted": False},
        # one decoded token's residual join
        {"name": "norm_token", "op": "norm", "T": 1, "d": 1536, "back": False, "stream": "bf16", "post": True,
         "gate": "none", "res_scale": 1.0, "branch_scale": 1.0},
        # a large batch on a 32-bit residual stream
        {"name": "norm_forward_large", "op": "norm", "T": 32768, "d": 4096, "back": False, "stream": "f32",
         "post": True, "gate": "shared", "res_scale": 1.0, "branch_scale": 0.5},
        # the training step of the ~1B student: norm after the branch, one learned gate per channel
        {"name": "norm_backward_1b", "op": "norm", "T": 8192, "d": 1536, "back": True, "stream": "bf16", "post": True,
         "gate": "shared", "res_scale": 1.0, "branch_scale": 1.0},
        # odd width, a gate for every token, scaled residual on a 32-bit stream
        {"name": "norm_backward_odd", "op": "norm", "T": 1000, "d": 1027, "back": True, "stream": "f32", "post": False,
         "gate": "token", "res_scale": 0.75, "branch_scale": 1.0},
        # one decoded token through the down projection, added to the residual stream
        {"name": "linear_token", "op": "linear", "M": 1, "N": 1536, "K": 6144, "back": False, "act": "none",
         "bias": True, "residual": True},
        # up projection of a packed row, pre-activation kept for the backward
        {"name": "linear_forward_up", "op": "linear", "M": 8192, "N": 6144, "K": 1536, "back": False,
         "act": "gelu_tanh", "bias": True, "residual": False},
        # ragged in every extent
        {"name": "linear_forward_odd", "op": "linear", "M": 333, "N": 1001, "K": 1000, "back": False, "act": "silu",
         "bias": True, "residual": True},
        # backward of the wide up projection (d = 4096)
        {"name": "linear_backward_up", "op": "linear", "M": 8192, "N": 16384, "K": 4096, "back": True,
         "act": "gelu_tanh", "bias": True, "residual": False},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("ce", "norm", "linear"))
    while True:
        if op == "ce":
            c = {"op": op, "T": _log_int(rng, 1, 8192), "d": 64 * _log_int(rng, 1, 64), "V": _log_int(rng, 500, 151936),
                 "tau": rng.choice((1.0, 1.0, 0.7, 2.0)), "step": rng.random() < 0.7, "masked": rng.random() < 0.7,
                 "weighted": rng.random() < 0.4}
            if c["T"] * c["d"] * c["V"] <= 8192 * 1536 * 151936 and c["T"] * c["V"] <= 8192 * 151936:
                return c
        elif op == "norm":
            c = {"op": op, "T": _log_int(rng, 1, 65536), "d": _log_int(rng, 64, 8192), "back": rng.random() < 0.6,
                 "stream": rng.choice(("bf16", "f32")), "post": rng.random() < 0.6,
                 "gate": rng.choice(("none", "shared", "token")), "res_scale": rng.choice((1.0, 0.75)),
                 "branch_scale": rng.choice((1.0, 0.5))}
            if c["T"] * c["d"] <= 20000 * 4096:
                return c
        else:
            c = {"op": op, "M": _log_int(rng, 1, 8192), "N": _log_int(rng, 64, 16384), "K": _log_int(rng, 64, 16384),
                 "back": rng.random() < 0.5, "act": rng.choice(ACTS), "bias": rng.random() < 0.7,
                 "residual": False}
            c["residual"] = not c["back"] and rng.random() < 0.5
            if c["M"] * c["N"] * c["K"] <= 8192 * 16384 * 4096:
                return c


# ------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------
def _rows(rows, cols, std, g, dtype=torch.bfloat16):
    """[rows, cols] normal values whose rows start on 16-byte boundaries (a multiple of 8 elements apart)."""
    ld = (cols + 7) // 8 * 8
    buf = torch.empty((rows, ld), dtype=dtype, device=DEV)
    step = max(1, (1 << 27) // ld)
    for a in range(0, rows, step):
        buf[a:a + step] = (torch.randn((min(step, rows - a), ld), generator=g, device=DEV) * std).to(dtype)
    return buf[:, :cols]


def _prepare_ce(c, g):
    T, d, V = c["T"], c["d"], c["V"]
    hidden, weight = _rows(T, d, 1.0, g), _rows(V, d, 0.02, g)
    labels = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    # a student that has learned something: the label's logit is raised by 0 to 12
    w_y = weight[labels.long()].float()
    up = 12.0 * torch.rand((T, 1), generator=g, device=DEV) * c["tau"]
    hidden.copy_((hidden.float() + up * w_y / w_y.square().sum(1, keepdim=True)).to(torch.bfloat16))
    s = {"case": c, "hidden": hidden, "weight": weight, "labels": labels, "mask": None, "tw": None}
    if c["masked"]:
        at = torch.arange(T, device=DEV)
        s["mask"] = (at % SEG >= PROMPT).to(torch.uint8)
        labels[SEG - 1::SEG] = IGNORE         # the last token of a segment predicts nothing
    if c["weighted"]:
        s["tw"] = torch.rand(T, generator=g, device=DEV) * 2.0
    s["grad_scale"] = 1.0 / max(1, _n_loss(c))
    return s


def _n_loss(c):
    """Tokens that carry loss."""
    if not c["masked"]:
        return c["T"]
    full, rest = divmod(c["T"], SEG)
    return full * (SEG - PROMPT - 1) + max(0, rest - PROMPT)


def _prepare_norm(c, g):
    T, d = c["T"], c["d"]
    sd = torch.float32 if c["stream"] == "f32" else torch.bfloat16
    s = {"case": c, "x": _rows(T, d, 1.5, g), "residual": _rows(T, d, 2.0, g, sd),
         "w_post": (1.0 + 0.2 * torch.randn(d, generator=g, device=DEV)) if c["post"] else None,
         "w_pre": 1.0 + 0.2 * torch.randn(d, generator=g, device=DEV), "gate": None, "eps": 1e-6}
    if c["gate"] == "shared":
        s["gate"] = (0.5 + 0.3 * torch.randn(d, generator=g, device=DEV)).to(torch.bfloat16)
    elif c["gate"] == "token":
        s["gate"] = _rows(T, d, 0.5, g)
    if c["back"]:
        # what the forward saved, and the gradients that arrive: at y, and at h from the blocks behind
        h = _rows(T, d, 2.0, g, sd)
        h.copy_((c["res_scale"] * s["residual"].float() + c["branch_scale"] * s["x"].float()).to(sd))
        s["h"], s["dy"], s["dh"] = h, _rows(T, d, 1e-2, g), _rows(T, d, 1e-2, g, sd)
    return s


def _prepare_linear(c, g):
    M, N, K = c["M"], c["N"], c["K"]
    s = {"case": c, "x": _rows(M, K, 1.0, g), "weight": _rows(N, K, 1.0 / math.sqrt(K), g), "bias": None,
         "residual": None, "z": None}
    if c["bias"]:
        s["bias"] = 0.2 * torch.randn(N, generator=g, device=DEV)
    if c["residual"]:
        s["residual"] = _rows(M, N, 2.0, g)
    if c["back"]:
        s["dy"] = _rows(M, N, 1e-2, g)
        if c["act"] != "none":
            s["z"] = _rows(M, N, 1.0, g)       # the pre-activation that the forward kept
    return s


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return {"ce": _prepare_ce, "norm": _prepare_norm, "linear": _prepare_linear}[case["op"]](case, g)


# ------------------------------------------------------------------------------------------------
# plain forms
# ------------------------------------------------------------------------------------------------
def _act(z, name):
    if name == "none":
        return z
    if name == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if name == "silu":
        return z * torch.sigmoid(z)
    if name == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))


def _dact(z, name):
    if name == "none":
        return torch.ones_like(z)
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "silu":
        s = torch.sigmoid(z)
        return s * (1.0 + z * (1.0 - s))
    if name == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    c = math.sqrt(2.0 / math.pi)
    t = torch.tanh(c * (z + 0.044715 * z * z * z))
    return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * c * (1.0 + 3 * 0.044715 * z * z)


def _plain_ce(s):
    c = s["case"]
    H, W = s["hidden"].float(), s["weight"].float()
    y = s["labels"].long()
    on = (y >= 0) & (y < c["V"])
    if s["mask"] is not None:
        on = on & (s["mask"] != 0)
    z = H @ W.t()
    z.mul_(1.0 / c["tau"])
    top = z.max(dim=1, keepdim=True).values
    p = torch.exp(z - top)
    total = p.sum(1, keepdim=True)
    lse = (top + torch.log(total)).squeeze(1)
    at = torch.where(on, y, torch.zeros_like(y)).unsqueeze(1)
    zero = torch.zeros_like(lse)
    nll = torch.where(on, lse - z.gather(1, at).squeeze(1), zero)
    lse = torch.where(on, lse, zero)
    if not c["step"]:
        return nll, lse
    coef = torch.where(on, zero + 1.0, zero) if s["tw"] is None else torch.where(on, s["tw"], zero)
    del z
    p.mul_((coef * (s["grad_scale"] / c["tau"])).unsqueeze(1) / total)
    p.scatter_add_(1, at, -(coef * (s["grad_scale"] / c["tau"])).unsqueeze(1))
    return nll, lse, (p @ W).to(torch.bfloat16), (p.t() @ H).to(torch.bfloat16)


def _plain_norm(s):
    c = s["case"]
    x = s["x"].float()
    rx = torch.rsqrt(x.square().mean(1, keepdim=True) + s["eps"]) if c["post"] else None
    n = x * rx * s["w_post"] if c["post"] else x
    gate = None if s["gate"] is None else s["gate"].float()
    if not c["back"]:
        b = n if gate is None else n * gate
        h = c["res_scale"] * s["residual"].float() + c["branch_scale"] * b
        y = h * torch.rsqrt(h.square().mean(1, keepdim=True) + s["eps"]) * s["w_pre"]
        return h.to(s["residual"].dtype), y.to(torch.bfloat16)
    h, dy = s["h"].float(), s["dy"].float()
    rh = torch.rsqrt(h.square().mean(1, keepdim=True) + s["eps"])
    u = dy * s["w_pre"]
    dh = s["dh"].float() + rh * (u - h * (rh * rh) * (u * h).mean(1, keepdim=True))
    out = {"dresidual": (c["res_scale"] * dh).to(s["h"].dtype), "d_w_pre": (dy * h * rh).sum(0)}
    if gate is not None:
        dg = c["branch_scale"] * n * dh
        out["d_gate"] = dg.sum(0) if c["gate"] == "shared" else dg.to(torch.bfloat16)
    dn = c["branch_scale"] * dh if gate is None else c["branch_scale"] * dh * gate
    if c["post"]:
        out["d_w_post"] = (dn * x * rx).sum(0)
        v = dn * s["w_post"]
        dn = rx * (v - x * (rx * rx) * (v * x).mean(1, keepdim=True))
    out["dx"] = dn.to(torch.bfloat16)
    return out


def _plain_linear(s):
    c = s["case"]
    x, w = s["x"].float(), s["weight"].float()
    if not c["back"]:
        z = x @ w.t()
        if s["bias"] is not None:
            z = z + s["bias"]
        y = _act(z, c["act"])
        if s["residual"] is not None:
            y = y + s["residual"].float()
        y = y.to(torch.bfloat16)
        return y if c["act"] == "none" else (y, z.to(torch.bfloat16))
    dz = s["dy"].float()
    if c["act"] != "none":
        dz = dz * _dact(s["z"].float(), c["act"])
    out = {"dx": (dz @ w).to(torch.bfloat16), "dw": (dz.t() @ x).to(torch.bfloat16)}
    if s["bias"] is not None:
        out["dbias"] = dz.sum(0)
    return out


# ------------------------------------------------------------------------------------------------
# the package's calls
# ------------------------------------------------------------------------------------------------
def _own_ce(s):
    from paper_2605_05940_b200 import binding as B
    c = s["case"]
    out = B.npd_cross_entropy(s["hidden"], s["weight"], s["labels"], loss_mask=s["mask"], token_weight=s["tw"],
                              temperature=c["tau"], grad_scale=s["grad_scale"], grads=c["step"])
    return out if c["step"] else out[:2]


def _own_norm(s):
    from paper_2605_05940_b200 import binding as B
    c = s["case"]
    how = dict(gate=s["gate"], post_weight=s["w_post"], pre_weight=s["w_pre"], post_norm=c["post"], eps=s["eps"],
               residual_scale=c["res_scale"], branch_scale=c["branch_scale"])
    if not c["back"]:
        return B.npd_norm_fwd(s["x"], s["residual"], **how)
    dx, dres, d_post, d_pre, d_gate = B.npd_norm_bwd(s["dy"], s["h"], s["x"], dh=s["dh"], **how)
    out = {"dresidual": dres, "d_w_pre": d_pre, "dx": dx}
    if c["post"]:
        out["d_w_post"] = d_post
    if s["gate"] is not None:
        out["d_gate"] = d_gate
    return out


def _own_linear(s):
    from paper_2605_05940_b200 import binding as B
    c = s["case"]
    act = {"none": B.NPD_ACT_NONE, "relu": B.NPD_ACT_RELU, "gelu": B.NPD_ACT_GELU,
           "gelu_tanh": B.NPD_ACT_GELU_TANH, "silu": B.NPD_ACT_SILU}[c["act"]]
    if not c["back"]:
        y, z = B.npd_linear_fwd(s["x"], s["weight"], bias=s["bias"], residual=s["residual"], activation=act,
                                want_preact=c["act"] != "none")
        return y if z is None else (y, z)
    dx, dw, db = B.npd_linear_bwd(s["dy"], s["x"], s["weight"], preact=s["z"], activation=act,
                                  want_dbias=s["bias"] is not None)
    out = {"dx": dx, "dw": dw}
    if db is not None:
        out["dbias"] = db
    return out


def run(state):
    op = state["case"]["op"]
    if own:
        return {"ce": _own_ce, "norm": _own_norm, "linear": _own_linear}[op](state)
    return {"ce": _plain_ce, "norm": _plain_norm, "linear": _plain_linear}[op](state)


# ------------------------------------------------------------------------------------------------
# work
# ------------------------------------------------------------------------------------------------
def work(case):
    c = case
    if c["op"] == "ce":
        n, T, d, V = _n_loss(c), c["T"], c["d"], c["V"]
        b = 2 * n * d + 2 * V * d + 4 * T + (T if c["masked"] else 0) + (4 * T if c["weighted"] else 0) + 8 * T
        if c["step"]:
            b += 2 * T * d + 2 * V * d
        return {"bytes": b, "flops": max(1, n) * d * V * (6 if c["step"] else 2)}
    if c["op"] == "norm":
        n, e = c["T"] * c["d"], 4 if c["stream"] == "f32" else 2
        small = 4 * c["d"] * (2 if c["post"] else 1) + (2 * c["d"] if c["gate"] == "shared" else 0)
        gate = 2 * n if c["gate"] == "token" else 0
        if not c["back"]:
            return {"bytes": n * (2 + e + e + 2) + gate + small, "flops": 10 * n}
        # reads dy, h, dh, x; writes dx, dresidual and the small gradients
        reads_x = 2 if c["post"] or c["gate"] != "none" else 0
        return {"bytes": n * (2 + e + e + reads_x + 2 + e) + 2 * gate + 2 * small, "flops": 25 * n}
    M, N, K = c["M"], c["N"], c["K"]
    if not c["back"]:
        outs = 2 if c["act"] != "none" else 1
        b = 2 * (M * K + N * K + outs * M * N) + (4 * N if c["bias"] else 0) + (2 * M * N if c["residual"] else 0)
        return {"bytes": b, "flops": 2 * M * N * K}
    ins = 2 if c["act"] != "none" else 1
    return {"bytes": 2 * (ins * M * N + 2 * M * K + 2 * N * K) + (4 * N if c["bias"] else 0), "flops": 4 * M * N * K}


# ------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ------------------------------------------------------------------------------------------------
def _phi(z):
    """Standard normal distribution function and density."""
    return 0.5 * torch.special.erfc(-z / math.sqrt(2.0)), torch.exp(-z * z / 2.0) / math.sqrt(2.0 * math.pi)


def _exact_act(z, name):
    """Value and derivative of the activation."""
    if name == "none":
        return z, torch.ones_like(z)
    if name == "relu":
        return z.clamp(min=0.0), (z > 0).double()
    if name == "silu":
        q = 1.0 / (1.0 + torch.exp(-z))
        return z * q, q + z * q * (1.0 - q)
    if name == "gelu":
        cdf, pdf = _phi(z)
        return z * cdf, cdf + z * pdf
    k = math.sqrt(2.0 / math.pi)
    u = k * (z + 0.044715 * z ** 3)
    q = 1.0 / (1.0 + torch.exp(-2.0 * u))              # (1 + tanh u) / 2
    return z * q, q + 2.0 * z * q * (1.0 - q) * k * (1.0 + 3.0 * 0.044715 * z ** 2)


def _exact_ce(s):
    c = s["case"]
    T, d, V, tau = c["T"], c["d"], c["V"], c["tau"]
    lab = s["labels"].cpu().numpy()
    ok = (lab >= 0) & (lab < V)
    if s["mask"] is not None:
        ok &= s["mask"].cpu().numpy() != 0
    rows = torch.from_numpy(np.flatnonzero(ok)).to(DEV)
    W = s["weight"].double()
    nll, lse = (torch.zeros(T, dtype=torch.float64, device=DEV) for _ in range(2))
    dH = torch.zeros((T, d), dtype=torch.float64, device=DEV)
    dW = torch.zeros((V, d), dtype=torch.float64, device=DEV)
    for a in range(0, rows.numel(), 2048):
        r = rows[a:a + 2048]
        H = s["hidden"][r].double()
        logits = (H @ W.t()) / tau
        at = s["labels"][r].long()
        i = torch.arange(r.numel(), device=DEV)
        l = torch.logsumexp(logits, dim=1)
        lse[r], nll[r] = l, l - logits[i, at]
        if c["step"]:
            P = torch.exp(logits - l[:, None])
            P[i, at] -= 1.0
            k = s["grad_scale"] / tau * (torch.ones_like(l) if s["tw"] is None else s["tw"][r].double())
            P *= k[:, None]
            dH[r] = P @ W
            dW += P.t() @ H
    return (nll, lse, dH, dW) if c["step"] else (nll, lse)


def _exact_norm(s):
    c = s["case"]
    T, d = c["T"], c["d"]
    wq = s["w_pre"].double()
    wp = s["w_post"].double() if c["post"] else None
    sums = {k: torch.zeros(d, dtype=torch.float64, device=DEV) for k in ("d_w_pre", "d_w_post", "d_gate")}
    got = {}

    def put(name, a, v):
        got.setdefault(name, torch.empty((T, d), dtype=torch.float64, device=DEV))[a:a + v.shape[0]] = v

    for a in range(0, T, 8192):
        cut = slice(a, min(T, a + 8192))
        x = s["x"][cut].double()
        rms = torch.sqrt((x * x).sum(1, keepdim=True) / d + s["eps"])
        xn = x / rms if c["post"] else x
        n = xn * wp if c["post"] else xn
        gate = 1.0 if s["gate"] is None else (s["gate"][cut] if c["gate"] == "token" else s["gate"]).double()
        if not c["back"]:
            h = c["res_scale"] * s["residual"][cut].double() + c["branch_scale"] * gate * n
            put("h", a, h)
            put("y", a, h / torch.sqrt((h * h).sum(1, keepdim=True) / d + s["eps"]) * wq)
            continue
        h, dy = s["h"][cut].double(), s["dy"][cut].double()
        rh = torch.sqrt((h * h).sum(1, keepdim=True) / d + s["eps"])
        hn = h / rh
        t = dy * wq
        dh = s["dh"][cut].double() + (t - hn * ((t * hn).sum(1, keepdim=True) / d)) / rh
        put("dresidual", a, c["res_scale"] * dh)
        sums["d_w_pre"] += (dy * hn).sum(0)
        db = c["branch_scale"] * dh
        if c["gate"] == "token":
            put("d_gate", a, db * n)
        elif c["gate"] == "shared":
            sums["d_gate"] += (db * n).sum(0)
        dn = db * gate
        if c["post"]:
            sums["d_w_post"] += (dn * xn).sum(0)
            t = dn * wp
            dn = (t - xn * ((t * xn).sum(1, keepdim=True) / d)) / rms
        put("dx", a, dn)
    if not c["back"]:
        return got["h"], got["y"]
    out = {"dresidual": got["dresidual"], "d_w_pre": sums["d_w_pre"], "dx": got["dx"]}
    if c["post"]:
        out["d_w_post"] = sums["d_w_post"]
    if c["gate"] != "none":
        out["d_gate"] = got["d_gate"] if c["gate"] == "token" else sums["d_gate"]
    return out


def _exact_linear(s):
    c = s["case"]
    W = s["weight"].double()
    if not c["back"]:
        z = torch.einsum("mk,nk->mn", s["x"].double(), W)
        if s["bias"] is not None:
            z = z + s["bias"].double()
        y = _exact_act(z, c["act"])[0]
        if s["residual"] is not None:
            y = y + s["residual"].double()
        return y if c["act"] == "none" else (y, z)
    dx = torch.empty((c["M"], c["K"]), dtype=torch.float64, device=DEV)
    dw = torch.zeros((c["N"], c["K"]), dtype=torch.float64, device=DEV)
    db = torch.zeros(c["N"], dtype=torch.float64, device=DEV)
    for a in range(0, c["M"], 4096):
        cut = slice(a, min(c["M"], a + 4096))
        g = s["dy"][cut].double()
        if c["act"] != "none":
            g = g * _exact_act(s["z"][cut].double(), c["act"])[1]
        dx[cut] = g @ W
        dw += g.t() @ s["x"][cut].double()
        db += g.sum(0)
    out = {"dx": dx, "dw": dw}
    if s["bias"] is not None:
        out["dbias"] = db
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return {"ce": _exact_ce, "norm": _exact_norm, "linear": _exact_linear}[case["op"]](s)
