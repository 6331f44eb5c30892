"""Timed cases of the operators that stand around the FP4 linears of a policy model.

Five kinds of pass ("op"), each one call of the package's public entry points:

* ``norm``       the residual update after a block with the norms around it: the block's output
                 is normalised, gated, scaled and added to the residual stream, and the result
                 is normalised for the next block's linears;
* ``norm_bwd``   its gradients;
* ``matvec``     a few tokens (1 to 16) times 4-bit weights with group scales;
* ``logprob``    log probabilities of given tokens under the policy's logits, with the entropy
                 and the top alternatives;
* ``logprob_bwd``  the gradient of the logits.

``run`` computes them in plain torch operations in float32, or, with ``own`` set, through the
package.  ``exact`` computes them in float64.  Inputs are drawn on the GPU from the seed.
"""
import math

import torch

own = False

EPS = 1e-6
INF = float("inf")


# ------------------------------------------------------------------------------------------
# cases
# ------------------------------------------------------------------------------------------
def _norm(name, op, m, d, h="bf16", y="f32", dx="f32", dy="bf16", post=True, gate="none", pre=True, save=True, pad=0):
    c = {"op": op, "m": m, "d": d, "h": h, "y": y, "dx": dx, "dy": dy, "post": post, "gate": gate, "pre": pre,
         "save": save, "pad": pad}
    return {"name": name, **c} if name else c


def _matvec(name, m, d, n, fmt, out="f32"):
    c = {"op": "matvec", "m": m, "d": d, "n": n, "fmt": fmt, "out": out}
    return {"name": name, **c} if name else c


def _logprob(name, op, m, v, x="f32", top=0, temp=1.0, ignored=0.0, banned=0.0, out="bf16", ent=True, pad=0):
    c = {"op": op, "m": m, "v": v, "x": x, "top": top, "temp": temp, "ignored": ignored, "banned": banned, "out": out,
         "ent": ent, "pad": pad}
    return {"name": name, **c} if name else c


def listed():
    return [
        # one token being decoded: the o projection's output joins the stream, the MLP's input norm
        _norm("norm_m1_d2048", "norm", 1, 2048, post=False, save=False),
        # a full batch of prompt tokens, norms on both sides of the block and a learned channel gate
        _norm("norm_m8192_d3584_gate", "norm", 8192, 3584, gate="channel"),
        # training: a small micro batch of a plain pre-norm model
        _norm("norm_bwd_m256_d2048", "norm_bwd", 256, 2048, post=False),
        # training: a full batch of tokens with both norms and the channel gate
        _norm("norm_bwd_m8192_d3584_gate", "norm_bwd", 8192, 3584, gate="channel"),
        # the last sequence of a rollout batch: a qkv projection for one token
        _matvec("matvec_m1_qkv_mxfp4", 1, 2048, 2560, "mxfp4"),
        # the last few sequences: the widest linear of the large block
        _matvec("matvec_m4_gateup_hif4", 4, 3584, 37888, "hif4"),
        # sixteen sequences: a down projection handed on in bf16
        _matvec("matvec_m16_down_hif4", 16, 11008, 2048, "hif4", out="bf16"),
        # one decoded token: its log probability, the entropy and twenty alternatives
        _logprob("logprob_m1_v131072_top20", "logprob", 1, 131072, top=20, temp=0.7),
        # a rollout batch with part of the vocabulary banned and five alternatives a token
        _logprob("logprob_m256_v131072_top5", "logprob", 256, 131072, top=5, banned=0.02),
        # training: packed responses of a micro batch, prompt tokens without a target, odd sizes
        _logprob("logprob_m2047_v100003", "logprob", 2047, 100003, x="bf16", ignored=0.2),
        # training: the logits' gradient, an odd and small one, and a micro batch of tokens
        _logprob("logprob_bwd_m63_v32003", "logprob_bwd", 63, 32003, x="bf16", ignored=0.1),
        _logprob("logprob_bwd_m1024_v131072", "logprob_bwd", 1024, 131072, ignored=0.2),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: a kind by lot, sizes spread over their ranges by their logarithm."""
    op = rng.choice(("norm", "norm", "norm_bwd", "norm_bwd", "matvec", "matvec", "logprob", "logprob", "logprob_bwd"))
    while True:
        if op in ("norm", "norm_bwd"):
            m, d = _log_int(rng, 1, 8192), _log_int(rng, 64, 16384)
            if rng.random() < 0.5:  # half of the widths as models have them
                d = max(64, d // 64 * 64)
            c = _norm(None, op, m, d, rng.choice(("bf16", "bf16", "f32")), rng.choice(("bf16", "f32", "f32")),
                      rng.choice(("bf16", "f32", "f32")), rng.choice(("bf16", "bf16", "f32")), rng.random() < 0.5,
                      rng.choice(("none", "channel", "token")), op == "norm_bwd" or rng.random() < 0.9,
                      rng.random() < 0.6, rng.choice((0, 0, 0, 1, 8, 40)))
            if m * d <= 8192 * 3584:
                return c
        elif op == "matvec":
            m, d, n = rng.randint(1, 16), 64 * _log_int(rng, 1, 296), _log_int(rng, 1, 40000)
            if n * d <= 37888 * 3584:
                return _matvec(None, m, d, n, rng.choice(("mxfp4", "hif4")), rng.choice(("f32", "f32", "bf16")))
        else:
            m, v = _log_int(rng, 1, 8192), _log_int(rng, 500, 160000)
            x = rng.choice(("f32", "bf16"))
            c = _logprob(None, op, m, v, x, rng.choice((0, 0, 1, 5, 20, 32)) if op == "logprob" else 0,
                         rng.choice((1.0, 1.0, 0.7, 1.3)), rng.choice((0.0, 0.1, 0.5)),
                         rng.choice((0.0, 0.02, 0.3)), rng.choice(("bf16", "bf16", "f32")), rng.random() < 0.6,
                         rng.choice((0, 0, 1, 8, 61)))
            if work(c)["bytes"] <= 700e6:
                return c


SIZE = {"bf16": 2, "f32": 4}
DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}


def work(c):
    m = c["m"]
    if c["op"] == "norm":
        d = c["d"]
        row = 2 * SIZE[c["h"]] + SIZE[c["y"]] + (2 if c["pre"] else 0)
        vec = 2 * (c["post"] + c["pre"] + (c["gate"] == "channel"))
        return {"bytes": m * d * row + d * vec + m * 8 * c["save"], "flops": 10 * m * d}
    if c["op"] == "norm_bwd":
        d = c["d"]
        row = 3 * SIZE[c["h"]] + SIZE[c["dx"]] + SIZE[c["dy"]]
        needs_y = c["post"] or c["gate"] != "none"
        row += SIZE[c["y"]] if needs_y else 0
        vec = 6 * (c["post"] + c["pre"] + (c["gate"] == "channel"))
        return {"bytes": m * d * row + d * vec + m * 8, "flops": 20 * m * d}
    if c["op"] == "matvec":
        d, n = c["d"], c["n"]
        bits = 4.25 if c["fmt"] == "mxfp4" else 4.5
        return {"bytes": int(n * d * bits / 8) + 2 * m * d + SIZE[c["out"]] * m * n, "flops": 2 * m * n * d}
    # the logits of a row without a target need not be read
    live = m - round(m * c["ignored"])
    v = c["v"]
    if c["op"] == "logprob":
        return {"bytes": live * v * SIZE[c["x"]] + m * (8 + 16 + 8 * c["top"]), "flops": 6 * live * v}
    return {"bytes": live * v * SIZE[c["x"]] + m * v * SIZE[c["out"]] + m * 28, "flops": 8 * live * v}


# ------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------
def _generator(c, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * seed + 7919 * ("norm", "norm_bwd", "matvec", "logprob", "logprob_bwd").index(c["op"]) + 1)
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _padded(x, dtype, pad):
    """x in that type, its rows `pad` elements further apart than they are long."""
    m, d = x.shape
    buf = torch.zeros((m, d + pad), dtype=dtype, device="cuda")
    buf[:, :d] = x
    return buf[:, :d]


def _norm_inputs(c, seed):
    g = _generator(c, seed)
    m, d = c["m"], c["d"]
    scale = 1 + 20 * (torch.rand(d, generator=g, device="cuda") < 0.01)  # a few outlier channels
    s = {"h": _padded(_randn(g, m, d) * scale, DTYPE[c["h"]], c["pad"]),
         "y": _padded(_randn(g, m, d) * 0.5, DTYPE[c["y"]], c["pad"]),
         "gamma_post": None, "gamma_pre": None, "gate": None, "alpha": 0.5 if c["post"] else 1.0}
    if c["post"]:
        s["gamma_post"] = (1 + 0.2 * _randn(g, d)).bfloat16()
    if c["pre"]:
        s["gamma_pre"] = (1 + 0.2 * _randn(g, d)).bfloat16()
    if c["gate"] == "channel":
        s["gate"] = (0.5 + 0.2 * _randn(g, d)).bfloat16()
    elif c["gate"] == "token":
        s["gate"] = torch.sigmoid(_randn(g, m, 1))
    if c["op"] == "norm_bwd":
        # h is the stream after the forward; the forward's factors come with it
        s["rstd"] = torch.stack([_rstd(s["y"].double()).float() if c["post"] else torch.zeros(m, device="cuda"),
                                 _rstd(s["h"].double()).float() if c["pre"] else torch.zeros(m, device="cuda")])
        s["dx"] = _padded(_randn(g, m, d) * 1e-2, DTYPE[c["dx"]], c["pad"])
        s["dh"] = _padded(_randn(g, m, d) * 1e-2, DTYPE[c["h"]], c["pad"])
    return s


def _rstd(x):
    return 1 / torch.sqrt((x * x).mean(1) + EPS)


def _matvec_inputs(c, seed):
    g = _generator(c, seed)
    m, d, n = c["m"], c["d"], c["n"]
    s = {"x": _randn(g, m, d).bfloat16()}
    # codes of normal weights (sign and the magnitude's 3-bit code) with the scales of rows about
    # 0.02 in size
    w = _randn(g, n, d)
    code = (w.abs() * 2.5).round_().clamp_(max=7).to(torch.uint8) + 8 * (w < 0).to(torch.uint8)
    s["codes"] = code[:, 0::2] + 16 * code[:, 1::2]
    if c["fmt"] == "mxfp4":
        s["scales"] = 127 - 6 - torch.randint(0, 3, (n, d // 32), generator=g, device="cuda").to(torch.uint8)
    else:
        level1 = 4 * (31 - 6) + torch.randint(-4, 4, (n, d // 64), generator=g, device="cuda")
        level23 = torch.randint(0, 1 << 24, (n, d // 64), generator=g, device="cuda")
        s["scales"] = (level1 | (level23 << 8)).to(torch.int64)
        s["scales"] = torch.where(s["scales"] >= 1 << 31, s["scales"] - (1 << 32), s["scales"]).to(torch.int32)
    return s


def _logprob_inputs(c, seed):
    g = _generator(c, seed)
    m, v = c["m"], c["v"]
    x = _randn(g, m, v).mul_(2.0)
    # a peaked next token in most rows, as a trained policy has
    peak = torch.randint(0, v, (m,), generator=g, device="cuda")
    x[torch.arange(m, device="cuda"), peak] += 4 + 12 * torch.rand(m, generator=g, device="cuda")
    if c["banned"]:
        banned = torch.rand(v, generator=g, device="cuda") < c["banned"]
        x[:, banned] = -INF
    x = _padded(x, DTYPE[c["x"]], c["pad"])
    other = torch.randint(0, v, (m,), generator=g, device="cuda")
    target = torch.where(torch.rand(m, generator=g, device="cuda") < 0.7, peak, other)
    # targets are sampled tokens, so never banned ones: the row's largest logit instead
    best = x.float().argmax(1)
    chosen = x[torch.arange(m, device="cuda"), target].float()
    target = torch.where(chosen == -INF, best, target)
    if c["ignored"]:  # the first tokens of a packed batch: a prompt, which has no targets
        target[: round(m * c["ignored"])] = -1
    s = {"x": x, "target": target, "temp": c["temp"]}
    if c["op"] == "logprob_bwd":
        stats = torch.empty((m, 3), dtype=torch.float32, device="cuda")
        for i in range(0, m, 256):
            stats[i:i + 256] = _logprob_exact(x[i:i + 256], target[i:i + 256], c["temp"])["stats"].float()
        s["stats"] = stats
        s["dlogp"] = _randn(g, m) / m
        s["dentropy"] = _randn(g, m) * 0.01 / m if c["ent"] else None
    return s


def prepare(c, seed):
    make = {"norm": _norm_inputs, "norm_bwd": _norm_inputs, "matvec": _matvec_inputs, "logprob": _logprob_inputs,
            "logprob_bwd": _logprob_inputs}[c["op"]]
    return {"case": c, **make(c, seed)}


# ------------------------------------------------------------------------------------------
# the plain forms
# ------------------------------------------------------------------------------------------
def _plain_norm(c, s):
    h, y = s["h"].float(), s["y"].float()
    m = c["m"]
    zero = torch.zeros(m, device="cuda")
    r_post = r_pre = zero
    if c["post"]:
        r_post = _rstd(y)
        y = y * r_post[:, None] * s["gamma_post"].float()
    if s["gate"] is not None:
        y = y * s["gate"].float()
    h_out = (h + s["alpha"] * y).to(DTYPE[c["h"]])
    x = None
    if c["pre"]:
        r_pre = _rstd(h_out.float())
        x = (h_out.float() * r_pre[:, None] * s["gamma_pre"].float()).bfloat16()
    return {"h": h_out, "x": x, "rstd": torch.stack([r_post, r_pre]) if c["save"] else None}


def _plain_norm_bwd(c, s):
    h, y, dx, e = s["h"].float(), s["y"].float(), s["dx"].float(), s["dh"].float()
    r_post, r_pre = s["rstd"][0][:, None], s["rstd"][1][:, None]
    out = {"dgamma_post": None, "dgamma_pre": None, "dgate": None}
    if c["pre"]:
        hn = h * r_pre
        u = dx * s["gamma_pre"].float()
        e = e + r_pre * (u - hn * (u * hn).mean(1, keepdim=True))
        out["dgamma_pre"] = (dx * hn).sum(0)
    yn = y * r_post if c["post"] else y
    t = yn * s["gamma_post"].float() if c["post"] else yn
    dt = s["alpha"] * e
    if s["gate"] is not None:
        out["dgate"] = (dt * t).sum(0) if c["gate"] == "channel" else (dt * t).sum(1, keepdim=True)
        dt = dt * s["gate"].float()
    dy = dt
    if c["post"]:
        out["dgamma_post"] = (dt * yn).sum(0)
        v = dt * s["gamma_post"].float()
        dy = r_post * (v - yn * (v * yn).mean(1, keepdim=True))
    return {"dh": e.to(DTYPE[c["h"]]), "dy": dy.to(DTYPE[c["dy"]]), **out}


def _weights(c, s, dtype):
    """The values of the codes: MXFP4 E2M1 times 2^(scale - 127); HiF4 k / 4 times the level-1
    scale, halved by the set bits of its group of 8 and of its group of 4."""
    n, d = c["n"], c["d"]
    code = torch.stack([s["codes"] & 15, s["codes"] >> 4], 2).reshape(n, d).long()
    if c["fmt"] == "mxfp4":
        mags = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6], dtype=dtype, device="cuda")
        scale = torch.exp2(s["scales"].to(dtype) - 127).repeat_interleave(32, 1)
    else:
        mags = torch.arange(8, dtype=dtype, device="cuda") / 4
        sc = s["scales"].long()
        level1 = torch.exp2(((sc >> 2) & 63).to(dtype) - 31) * (1 + (sc & 3).to(dtype) / 4)
        two = (sc[:, :, None] >> (8 + torch.arange(8, device="cuda"))) & 1
        four = (sc[:, :, None] >> (16 + torch.arange(16, device="cuda"))) & 1
        shift = (two.repeat_interleave(2, 2) + four).reshape(n, d // 4).to(dtype)
        scale = level1.repeat_interleave(16, 1) * torch.exp2(-shift)
        scale = scale.repeat_interleave(4, 1)
    value = mags[code & 7] * scale
    return torch.where(code >= 8, -value, value)


def _plain_matvec(c, s):
    return {"y": (s["x"].float() @ _weights(c, s, torch.float32).t()).to(DTYPE[c["out"]])}


def _plain_logprob(c, s):
    x, target, t = s["x"].float(), s["target"], s["temp"]
    m, v = x.shape
    live = target >= 0
    mx = x.max(1, keepdim=True).values
    z = (x - mx) / t
    e = torch.exp(z)
    total = e.sum(1)
    log_sum = torch.log(total)
    entropy = log_sum - torch.where(e > 0, e * z, 0.0).sum(1) / total
    logp = z.gather(1, target.clamp(min=0)[:, None])[:, 0] - log_sum
    stats = torch.stack([mx[:, 0], log_sum, entropy], 1)
    out = {"logp": torch.where(live, logp, 0.0), "stats": torch.where(live[:, None], stats, 0.0)}
    k = c["top"]
    if k:
        val, idx = torch.sort(x, dim=1, descending=True, stable=True)
        val, idx = val[:, :k], idx[:, :k]
        gone = (val == -INF) | ~live[:, None]
        out["top_logp"] = torch.where(gone, -INF, (val - mx) / t - log_sum[:, None])
        out["top_index"] = torch.where(gone, -1, idx).int()
    return out


def _plain_logprob_bwd(c, s):
    x, target, t = s["x"].float(), s["target"], s["temp"]
    live = (target >= 0)[:, None]
    a = s["dlogp"][:, None]
    logp = (x - s["stats"][:, 0:1]) / t - s["stats"][:, 1:2]
    p = torch.exp(logp)
    g = -a * p
    if s["dentropy"] is not None:
        g = g - torch.where(p > 0, s["dentropy"][:, None] * p * (logp + s["stats"][:, 2:3]), 0.0)
    g.scatter_add_(1, target.clamp(min=0)[:, None], a)
    return {"dlogits": torch.where(live, g / t, 0.0).to(DTYPE[c["out"]])}


# ------------------------------------------------------------------------------------------
# the package's operators
# ------------------------------------------------------------------------------------------
def _own(c, s):
    import paper_2607_26515_amd as P
    op = c["op"]
    if op == "norm":
        h, x, rstd = P.block_norm(s["h"], s["y"], gamma_post=s["gamma_post"], gate=s["gate"], alpha=s["alpha"],
                                  gamma_pre=s["gamma_pre"], eps=EPS, save=c["save"])
        return {"h": h, "x": x, "rstd": rstd}
    if op == "norm_bwd":
        return P.block_norm_bwd(s["h"], s["rstd"], dx=s["dx"], dh=s["dh"], y=s["y"], gamma_post=s["gamma_post"],
                                gate=s["gate"], alpha=s["alpha"], gamma_pre=s["gamma_pre"], out=c["dy"])
    if op == "matvec":
        return {"y": P.matvec_w4a16(s["x"], s["codes"], s["scales"], c["fmt"], out=c["out"])}
    if op == "logprob":
        return P.token_logprobs(s["x"], s["target"], temperature=s["temp"], top_k=c["top"])
    return {"dlogits": P.token_logprobs_bwd(s["x"], s["target"], s["stats"], s["dlogp"], dentropy=s["dentropy"],
                                            temperature=s["temp"], out=c["out"])}


def run(state):
    c = state["case"]
    if own:
        return _own(c, state)
    return {"norm": _plain_norm, "norm_bwd": _plain_norm_bwd, "matvec": _plain_matvec, "logprob": _plain_logprob,
            "logprob_bwd": _plain_logprob_bwd}[c["op"]](c, state)


# ------------------------------------------------------------------------------------------
# in 64 bits, from the definitions
# ------------------------------------------------------------------------------------------
def _norm_exact(c, s):
    h, y = s["h"].double(), s["y"].double()
    m, d = h.shape
    r = torch.zeros((2, m), dtype=torch.float64, device="cuda")
    branch = y
    if c["post"]:
        r[0] = torch.rsqrt(y.pow(2).sum(1) / d + EPS)
        branch = torch.einsum("ij,i,j->ij", y, r[0], s["gamma_post"].double())
    if s["gate"] is not None:
        branch = branch * s["gate"].double()
    h_out = h + s["alpha"] * branch
    x = None
    if c["pre"]:  # the norm is that of the stored stream
        stored = h_out.to(DTYPE[c["h"]]).double()
        r[1] = torch.rsqrt(stored.pow(2).sum(1) / d + EPS)
        x = torch.einsum("ij,i,j->ij", stored, r[1], s["gamma_pre"].double())
    return {"h": h_out, "x": x, "rstd": r if c["save"] else None}


def _norm_bwd_exact(c, s):
    """Every gradient as a vector-Jacobian product of the normalised row n(z) = z r(z):
    J^T u = r (u - n <u, n> / d), with the forward's factors r as given."""
    m, d = s["h"].shape
    rp, rh = s["rstd"][0].double(), s["rstd"][1].double()

    def through_norm(u, n, r):
        return r[:, None] * (u - n * ((u * n).sum(1) / d)[:, None])

    e = s["dh"].double()
    out = {"dgamma_post": None, "dgamma_pre": None, "dgate": None}
    if c["pre"]:
        n, dx = s["h"].double() * rh[:, None], s["dx"].double()
        e = e + through_norm(dx * s["gamma_pre"].double()[None, :], n, rh)
        out["dgamma_pre"] = (n * dx).sum(0)
    y = s["y"].double()
    n = y * rp[:, None] if c["post"] else y
    gp = s["gamma_post"].double()[None, :] if c["post"] else 1.0
    gate = s["gate"].double() if s["gate"] is not None else 1.0
    if c["gate"] != "none":
        prod = s["alpha"] * e * n * gp
        out["dgate"] = prod.sum(0) if c["gate"] == "channel" else prod.sum(1, keepdim=True)
    dy = s["alpha"] * gate * e
    if c["post"]:
        out["dgamma_post"] = (dy * n).sum(0)
        dy = through_norm(dy * gp, n, rp)
    return {"dh": e, "dy": dy, **out}


def _matvec_exact(c, s):
    """Row by row of codes: each group's sum in 64 bits, times the group's scale."""
    n, d = c["n"], c["d"]
    x = s["x"].double()
    y = torch.empty((c["m"], n), dtype=torch.float64, device="cuda")
    for i in range(0, n, 4096):
        b = s["codes"][i:i + 4096].int()
        code = torch.empty((b.shape[0], d), dtype=torch.int32, device="cuda")
        code[:, 0::2], code[:, 1::2] = b & 0xF, b >> 4
        k, sign = (code & 7).double(), 1.0 - 2.0 * (code >> 3).double()
        if c["fmt"] == "mxfp4":  # E2M1: exponent k >> 1, mantissa k & 1, subnormal below 2
            ex = (code & 7) >> 1
            mag = torch.where(ex == 0, k / 2, torch.ldexp(1 + (code & 1).double() / 2, ex - 1))
            value = torch.ldexp((sign * mag).view(-1, d // 32, 32), s["scales"][i:i + 4096].int()[:, :, None] - 127)
        else:
            sc = s["scales"][i:i + 4096].long() & 0xFFFFFFFF
            pos = torch.arange(64, device="cuda")
            halve = ((sc[:, :, None] >> (8 + pos // 8)) & 1) + ((sc[:, :, None] >> (16 + pos // 4)) & 1)
            s1 = torch.ldexp((4 + (sc & 3)).double(), ((sc & 255) >> 2).int() - 33)
            value = torch.ldexp((sign * k / 4).view(-1, d // 64, 64) * s1[:, :, None], -halve.int())
        y[:, i:i + 4096] = x @ value.reshape(-1, d).t().contiguous()
    return {"y": y}


def _logprob_exact(x, target, t, k=0):
    x = x.double()
    live = target >= 0
    lse = torch.logsumexp(x / t, 1)
    mx = x.amax(1)
    logq = x / t - lse[:, None]
    q = torch.exp(logq)
    entropy = -torch.special.xlogy(q, q).sum(1)
    at = target.clamp(min=0)[:, None]
    out = {"logp": torch.where(live, logq.gather(1, at)[:, 0], 0.0),
           "stats": torch.where(live[:, None], torch.stack([mx, lse - mx / t, entropy], 1), 0.0)}
    if k:
        v = x.shape[1]
        order = torch.argsort(-x, dim=1, stable=True)[:, :k]
        val = logq.gather(1, order)
        gone = (val == -INF) | ~live[:, None]
        out["top_logp"] = val.masked_fill(gone, -INF)
        out["top_index"] = order.masked_fill(gone, -1).int()
    return out


def _logprob_bwd_exact(x, target, t, stats, a, b):
    x, stats = x.double(), stats.double()
    logq = (x - stats[:, 0:1]) / t - stats[:, 1:2]
    q = torch.exp(logq)
    hot = torch.zeros_like(q).scatter_(1, target.clamp(min=0)[:, None], 1.0)
    g = a.double()[:, None] * (hot - q)
    if b is not None:
        g = g - b.double()[:, None] * (torch.special.xlogy(q, q) + q * stats[:, 2:3])
    return (g / t) * (target >= 0)[:, None]


def exact(c, seed):
    s = prepare(c, seed)
    if c["op"] == "norm":
        return _norm_exact(c, s)
    if c["op"] == "norm_bwd":
        return _norm_bwd_exact(c, s)
    if c["op"] == "matvec":
        return _matvec_exact(c, s)
    parts = []
    for i in range(0, c["m"], 128):  # rows at a time: 64-bit copies of all logits would be large
        x, t = s["x"][i:i + 128], s["target"][i:i + 128]
        if c["op"] == "logprob":
            parts.append(_logprob_exact(x, t, s["temp"], c["top"]))
        else:
            b = None if s["dentropy"] is None else s["dentropy"][i:i + 128]
            parts.append({"dlogits": _logprob_bwd_exact(x, t, s["temp"], s["stats"][i:i + 128],
                                                        s["dlogp"][i:i + 128], b)})
    return {key: torch.cat([p[key] for p in parts]) for key in parts[0]}
