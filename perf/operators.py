"""The measured work of the operators that run and score a quantised model.

Behind the solve a layer is codes, scales and zeros.  Three operators use it: the
root-mean-square norm before a layer (with the residual's addition, and an 8-bit output
where the layer wants one), the product with the quantised weight (with bias, activation
and residual), and the log probabilities of given tokens at the end, with entropy and top
alternatives; the norm and the log probabilities have their gradients too, which give the
output-side samples of the Hessian factors.

``listed`` gives the fixed cases, ``draw`` more of the same ranges, ``prepare`` what a
program holds before the call, ``run`` one pass, ``work`` its unavoidable bytes and
flops, ``exact`` its outputs in 64 bits.  Layer sizes are those of the workloads here;
token counts run from one (a decoding step) to a few thousand.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn}
EPS = 1e-5
E4M3_MAX = 448.0


def listed():
    return [
        # one decoding step through a 4096 x 4096 projection, 4-bit groups of 128, into the residual stream
        {"name": "linear_1_token", "op": "linear", "t": 1, "m": 4096, "n": 4096, "bits": 4, "group": 128,
         "x": "bf16", "act": "none", "bias": False, "residual": True},
        # a small batch of decoding steps through an MLP's down-projection with 8-bit codes, ragged sides
        {"name": "linear_17_tokens_8_bits", "op": "linear", "t": 17, "m": 4099, "n": 11003, "bits": 8, "group": 0,
         "x": "bf16", "act": "none", "bias": True, "residual": False},
        # a prompt of 1000 tokens through an MLP's up-projection, 3-bit groups of 128
        {"name": "linear_1000_tokens", "op": "linear", "t": 1000, "m": 11008, "n": 4096, "bits": 3, "group": 128,
         "x": "bf16", "act": "silu", "bias": True, "residual": False},
        # calibration batches through the largest layer, 8-bit inputs, one grid a row
        {"name": "linear_4096_tokens_e4m3", "op": "linear", "t": 4096, "m": 28672, "n": 8192, "bits": 4, "group": 0,
         "x": "e4m3", "act": "gelu", "bias": False, "residual": False},
        # the norm of one decoding step, handing 8 bits to the next product
        {"name": "norm_1_row_e4m3", "op": "norm", "t": 1, "d": 4096, "x": "bf16", "y": "e4m3", "residual": True},
        # the norm of a calibration batch, an odd number of rows
        {"name": "norm_16381_rows", "op": "norm", "t": 16381, "d": 8192, "x": "bf16", "y": "bf16", "residual": True},
        # its gradient, few ragged rows in fp32 and many in bf16
        {"name": "norm_back_37_rows", "op": "norm_back", "t": 37, "d": 11003, "x": "f32", "residual": False},
        {"name": "norm_back_8192_rows", "op": "norm_back", "t": 8192, "d": 4096, "x": "bf16", "residual": True},
        # the log probability of one decoded token with its five best alternatives
        {"name": "logprob_1_token", "op": "logprob", "t": 1, "v": 32000, "x": "bf16", "top": 5, "masked": 0},
        # scoring two sequences of 2048 tokens over a large vocabulary whose last entries are padding
        {"name": "logprob_4095_tokens", "op": "logprob", "t": 4095, "v": 128256, "x": "bf16", "top": 20, "masked": 100},
        # gradients at the logits: a few fp32 rows of odd length, and a scored batch
        {"name": "logprob_back_64_tokens", "op": "logprob_back", "t": 64, "v": 50021, "x": "f32", "entropy": True,
         "masked": 0},
        {"name": "logprob_back_4096_tokens", "op": "logprob_back", "t": 4096, "v": 128256, "x": "bf16",
         "entropy": False, "masked": 0},
    ]


def _between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["linear", "linear", "norm", "norm_back", "logprob", "logprob_back"])
    if op == "linear":
        bits = rng.choice([2, 3, 4, 4, 8])
        group = rng.choice([0, 0, 32, 64, 128])
        t, m, n = _between(rng, 1, 4096), _between(rng, 128, 28672), _between(rng, 128, 11008)
        if group:
            n = max(1, n // group) * group
        elif rng.random() < 0.5:
            n = n // 128 * 128
        t = min(t, 4096 * 28672 * 8192 // (m * n))
        return {"op": op, "t": t, "m": m, "n": n, "bits": bits, "group": group, "x": rng.choice(["bf16", "e4m3"]),
                "act": rng.choice(["none", "relu", "silu", "gelu"]), "bias": rng.random() < 0.5,
                "residual": rng.random() < 0.5}
    if op in ("norm", "norm_back"):
        d = _between(rng, 64, 16384)
        t = _between(rng, 1, min(16384, (16381 * 8192 if op == "norm" else 8192 * 4096) // (2 * d)))
        if rng.random() < 0.5:
            d = max(64, d // 64 * 64)
        case = {"op": op, "t": t, "d": d, "x": rng.choice(["bf16", "f32"]), "residual": rng.random() < 0.5}
        if op == "norm":
            case["y"] = rng.choice(["e4m3", case["x"]])
        return case
    v = _between(rng, 500, 128256)
    t = _between(rng, 1, min(4096, 4096 * 128256 // (2 * v)))
    case = {"op": op, "t": t, "v": v, "x": rng.choice(["bf16", "f32"]), "masked": rng.choice([0, v // 50])}
    if op == "logprob":
        case["top"] = rng.choice([0, 1, 5, 20, 32])
    else:
        case["entropy"] = rng.random() < 0.5
    return case


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _hidden(g, t, d):
    """Rows of a residual stream: uneven channels, a few of them large."""
    chan = 0.5 + torch.rand(d, generator=g, device="cuda")
    chan[torch.randint(0, d, (max(1, d // 512),), generator=g, device="cuda")] *= 8
    return torch.randn(t, d, generator=g, device="cuda") * chan


def _logits(g, case):
    x = 2.5 * torch.randn(case["t"], case["v"], generator=g, device="cuda")
    x[:, : max(1, case["v"] // 1000)] += 3.0     # frequent tokens
    if case["masked"]:
        x[:, case["v"] - case["masked"]:] = -math.inf
    return x.to(DTYPES[case["x"]])


def _targets(g, case):
    t = torch.randint(0, case["v"] - case["masked"], (case["t"],), generator=g, device="cuda")
    t[torch.rand(case["t"], generator=g, device="cuda") < 0.05] = -100     # positions that are not scored
    return t


def prepare(case, seed):
    g = _gen(seed)
    s = {"case": case}
    if case["op"] == "linear":
        t, m, n, group = case["t"], case["m"], case["n"], case["group"]
        qmax, G = 2 ** case["bits"] - 1, (n // group if group else 1)
        s["codes"] = torch.randint(0, qmax + 1, (m, n), generator=g, device="cuda", dtype=torch.uint8)
        s["scales"] = (0.5 + torch.rand(m, G, generator=g, device="cuda")) * (0.08 / qmax)
        s["zeros"] = torch.round((0.4 + 0.2 * torch.rand(m, G, generator=g, device="cuda")) * qmax)
        x = _hidden(g, t, n)
        s["x_scales"] = None
        if case["x"] == "e4m3":
            s["x_scales"] = x.abs().amax(1) / E4M3_MAX
            x = x / s["x_scales"][:, None]
        s["x"] = x.to(DTYPES[case["x"]])
        s["bias"] = 0.1 * torch.randn(m, generator=g, device="cuda") if case["bias"] else None
        s["residual"] = torch.randn(t, m, generator=g, device="cuda").bfloat16() if case["residual"] else None
        if own:     # a program keeps the weight laid out for its products
            import paper_2608_06291_gb300 as P
            s["weight"] = P.bakron_pack_weight(s["codes"], s["scales"], s["zeros"], qmax, group)
    elif case["op"] in ("norm", "norm_back"):
        t, d, dt = case["t"], case["d"], DTYPES[case["x"]]
        s["x"] = _hidden(g, t, d).to(dt)
        s["weight"] = (1 + 0.2 * torch.randn(d, generator=g, device="cuda")).to(dt)
        s["residual"] = torch.randn(t, d, generator=g, device="cuda").to(dt) if case["residual"] else None
        if case["op"] == "norm_back":     # the residual stream's own gradient joins the norm's
            s["dy"] = torch.randn(t, d, generator=g, device="cuda").to(dt)
    else:
        s["logits"], s["targets"] = _logits(g, case), _targets(g, case)
        if case["op"] == "logprob_back":
            s["dlogp"] = torch.randn(case["t"], generator=g, device="cuda")
            s["dentropy"] = 0.1 * torch.randn(case["t"], generator=g, device="cuda") if case["entropy"] else None
            x = s["logits"].float()     # what the forward pass left
            top = x.amax(1, keepdim=True)
            e = torch.exp(x - top)
            z = e.sum(1)
            s["lse"] = top[:, 0] + torch.log(z)
            s["entropy"] = torch.log(z) - torch.where(e > 0, e * (x - top), 0).sum(1) / z
    return s


def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    import paper_2608_06291_gb300 as P
    case = s["case"]
    if case["op"] == "linear":
        return P.bakron_linear(s["x"], s["weight"], x_scales=s["x_scales"], bias=s["bias"],
                               activation=case["act"], residual=s["residual"])
    if case["op"] == "norm":
        y, scales, total = P.bakron_rmsnorm(s["x"], s["weight"], EPS, residual=s["residual"],
                                            out_dtype=DTYPES[case["y"]])
        return {"y": y, "scales": scales, "sum": total}
    if case["op"] == "norm_back":
        dx, dw = P.bakron_rmsnorm_backward(s["dy"], s["x"], s["weight"], EPS, dsum=s["residual"])
        return {"dx": dx, "dw": dw}
    if case["op"] == "logprob":
        logp, entropy, lse, top_logp, top_ids = P.bakron_token_logprobs(s["logits"], s["targets"], case["top"])
        return {"logp": logp, "entropy": entropy, "lse": lse, "top_logp": top_logp, "top_ids": top_ids}
    return P.bakron_token_logprobs_backward(s["logits"], s["targets"], s["lse"], s["dlogp"],
                                            entropy=s["entropy"], dentropy=s["dentropy"])


def _act(v, name):
    if name == "relu":
        return torch.clamp(v, min=0)
    if name == "silu":
        return v / (1 + torch.exp(-v))
    if name == "gelu":
        return 0.5 * v * (1 + torch.erf(v * math.sqrt(0.5)))
    return v


def _plain(s):
    case = s["case"]
    if case["op"] == "linear":
        # the weight is held as codes; its values are formed within the call, as a program does
        # that has no room for both
        m, n = s["codes"].shape
        G = s["scales"].shape[1]
        w = s["codes"].float().view(m, G, n // G)
        w = ((w - s["zeros"][:, :, None]) * s["scales"][:, :, None]).view(m, n)
        y = s["x"].float() @ w.t()
        if s["x_scales"] is not None:
            y = y * s["x_scales"][:, None]
        if s["bias"] is not None:
            y = y + s["bias"]
        y = _act(y, case["act"])
        if s["residual"] is not None:
            y = y + s["residual"].float()
        return y.to(torch.bfloat16)
    if case["op"] == "norm":
        h = s["x"].float()
        if s["residual"] is not None:
            h = h + s["residual"].float()
        y = h * torch.rsqrt((h * h).mean(1, keepdim=True) + EPS) * s["weight"].float()
        scales = None
        if case["y"] == "e4m3":
            scales = y.abs().amax(1) / E4M3_MAX
            scales = torch.where(scales == 0, 1.0, scales)
            y = y / scales[:, None]
        return {"y": y.to(DTYPES[case["y"]]), "scales": scales,
                "sum": h.to(s["x"].dtype) if s["residual"] is not None else None}
    if case["op"] == "norm_back":
        h, dy, w = s["x"].float(), s["dy"].float(), s["weight"].float()
        r = torch.rsqrt((h * h).mean(1, keepdim=True) + EPS)
        c = (dy * w * h).mean(1, keepdim=True)
        dx = r * (dy * w - h * (r * r * c))
        if s["residual"] is not None:
            dx = dx + s["residual"].float()
        return {"dx": dx.to(s["x"].dtype), "dw": (dy * h * r).sum(0)}
    x, at = s["logits"].float(), s["targets"]
    scored = at >= 0
    if case["op"] == "logprob":
        top = x.amax(1, keepdim=True)
        e = torch.exp(x - top)
        z = e.sum(1)
        lse = top[:, 0] + torch.log(z)
        entropy = torch.log(z) - torch.where(e > 0, e * (x - top), 0).sum(1) / z
        logp = torch.where(scored, x.gather(1, at.clamp(min=0)[:, None])[:, 0] - lse, 0)
        out = {"logp": logp, "entropy": entropy, "lse": lse, "top_logp": None, "top_ids": None}
        if case["top"]:
            # ties go to the lowest index: one whole number of the value and the index
            bits = (x + 0.0).view(torch.int32)
            key = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).to(torch.int64)
            key = (key << 32) + torch.arange(x.shape[1] - 1, -1, -1, device=x.device)
            ids = x.shape[1] - 1 - (key.topk(case["top"], dim=1).values & 0xFFFFFFFF)
            out["top_logp"] = x.gather(1, ids) - lse[:, None]
            out["top_ids"] = ids.to(torch.int32)
        return out
    logp = x - s["lse"][:, None]
    p = torch.exp(logp)
    g = torch.where(scored, s["dlogp"], 0)
    d = -g[:, None] * p
    if s["dentropy"] is not None:
        d = d - torch.where(p > 0, s["dentropy"][:, None] * p * (logp + s["entropy"][:, None]), 0)
    d.scatter_add_(1, at.clamp(min=0)[:, None], g[:, None])
    return d.to(s["logits"].dtype)


def work(case):
    if case["op"] == "linear":
        t, m, n = case["t"], case["m"], case["n"]
        G = n // case["group"] if case["group"] else 1
        size = 1 if case["x"] == "e4m3" else 2
        read = m * n * (0.5 if case["bits"] <= 4 else 1) + 5 * m * G + t * n * size
        read += (4 * t if case["x"] == "e4m3" else 0) + (4 * m if case["bias"] else 0)
        read += 2 * t * m if case["residual"] else 0
        return {"bytes": read + 2 * t * m, "flops": 2.0 * t * m * n}
    if case["op"] in ("norm", "norm_back"):
        t, d = case["t"], case["d"]
        size = 2 if case["x"] == "bf16" else 4
        if case["op"] == "norm":
            out = {"bf16": 2, "f32": 4, "e4m3": 1}[case["y"]]
            scales = 4 * t if case["y"] == "e4m3" else 0
            return {"bytes": t * d * (size * (3 if case["residual"] else 1) + out) + size * d + scales,
                    "flops": 5.0 * t * d}
        return {"bytes": t * d * size * (4 if case["residual"] else 3) + (size + 4) * d, "flops": 11.0 * t * d}
    t, v = case["t"], case["v"]
    size = 2 if case["x"] == "bf16" else 4
    if case["op"] == "logprob":
        return {"bytes": t * v * size + t * (8 + 12 + 8 * case["top"]), "flops": 6.0 * t * v}
    return {"bytes": 2 * t * v * size + t * 20, "flops": 6.0 * t * v}


def _round_e4m3(v):
    """Nearest value of the 8-bit format (4 exponent bits from 2^-6, 3 of the fraction), ties to even."""
    e = torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6)))
    e = torch.where(v.abs() >= torch.exp2(e + 1), e + 1, e)
    step = torch.exp2(e - 3)
    return (torch.round(v / step) * step).clamp(-E4M3_MAX, E4M3_MAX)


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    if case["op"] == "linear":
        t, m, n = case["t"], case["m"], case["n"]
        x = s["x"].to(torch.float32).double()
        if s["x_scales"] is not None:
            x *= s["x_scales"].double()[:, None]
        y = torch.empty(t, m, dtype=torch.float64, device="cuda")
        group = case["group"] or n
        for i in range(0, m, 4096):
            w = s["codes"][i:i + 4096].double()
            w -= s["zeros"][i:i + 4096].double().repeat_interleave(group, 1)
            w *= s["scales"][i:i + 4096].double().repeat_interleave(group, 1)
            y[:, i:i + 4096] = x @ w.t()
        if s["bias"] is not None:
            y += s["bias"].double()
        acts = {"gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu, "relu": torch.relu}
        y = acts[case["act"]](y) if case["act"] in acts else y
        return y if s["residual"] is None else y + s["residual"].double()
    if case["op"] == "norm":
        h = s["x"].double()
        if s["residual"] is not None:
            h = h + s["residual"].double()
        y = h / torch.sqrt(h.square().sum(1, keepdim=True) / case["d"] + EPS) * s["weight"].double()
        scales = None
        if case["y"] == "e4m3":
            scales = y.abs().max(1).values / E4M3_MAX
            scales[scales == 0] = 1.0
            y = _round_e4m3(y / scales[:, None])
        return {"y": y, "scales": scales, "sum": h if s["residual"] is not None else None}
    if case["op"] == "norm_back":
        h, dy, w = s["x"].double(), s["dy"].double(), s["weight"].double()
        sigma = torch.sqrt(h.square().sum(1, keepdim=True) / case["d"] + EPS)
        xhat = h / sigma
        back = dy * w
        dx = (back - xhat * ((back * xhat).sum(1, keepdim=True) / case["d"])) / sigma
        if s["residual"] is not None:
            dx += s["residual"].double()
        return {"dx": dx, "dw": (dy * xhat).sum(0)}
    out = {k: [] for k in ("logp", "entropy", "lse", "top_logp", "d")}
    for i in range(0, case["t"], 512):
        x, at = s["logits"][i:i + 512].double(), s["targets"][i:i + 512]
        if case["op"] == "logprob":
            lse = torch.logsumexp(x, 1)
            logp = x - lse[:, None]
            out["lse"].append(lse)
            out["entropy"].append(-torch.special.xlogy(logp.exp(), logp.exp()).sum(1))
            out["logp"].append(torch.where(at >= 0, logp.gather(1, at.clamp(min=0)[:, None])[:, 0], 0.0))
            if case["top"]:
                out["top_logp"].append(logp.topk(case["top"], 1).values)
        else:
            logp = x - s["lse"][i:i + 512].double()[:, None]
            d = torch.zeros_like(x)
            d.scatter_(1, at.clamp(min=0)[:, None], 1.0)
            d -= logp.exp()
            d *= torch.where(at >= 0, s["dlogp"][i:i + 512].double(), 0.0)[:, None]
            if s["dentropy"] is not None:
                e = torch.special.xlogy(logp.exp(), logp.exp()) + logp.exp() * s["entropy"][i:i + 512].double()[:, None]
                d -= s["dentropy"][i:i + 512].double()[:, None] * e
            out["d"].append(d)
    if case["op"] == "logprob_back":
        return torch.cat(out["d"])
    return {"logp": torch.cat(out["logp"]), "entropy": torch.cat(out["entropy"]), "lse": torch.cat(out["lse"]),
            "top_logp": torch.cat(out["top_logp"]) if case["top"] else None, "top_ids": None}
