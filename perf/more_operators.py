"""The measured work of the operators that carry gradients back through a quantised model.

Behind the forward operators three things were missing on the way from a model's loss to
the output-side samples of each layer's Hessian factors.  The head: log probabilities of
given tokens straight from the hidden states and the head's weight, over a vocabulary so
large that logits are not kept, with the gradients at both.  The layer norm, which many models have in place of the
root-mean-square norm, with its gradients.  And the gradient of the product with a
quantised weight at its tokens, which hands the samples on to the layer before.

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
        # scoring one decoded token
        {"name": "head_1_token", "op": "head", "t": 1, "v": 32000, "d": 4096},
        # scoring a short ragged prompt with a small model
        {"name": "head_77_tokens", "op": "head", "t": 77, "v": 50021, "d": 1000},
        # scoring two sequences of 2048 tokens over a large vocabulary
        {"name": "head_4095_tokens", "op": "head", "t": 4095, "v": 128256, "d": 4096},
        # samples at the hidden states of a few tokens, the weight's gradient not wanted
        {"name": "head_back_64_tokens", "op": "head_back", "t": 64, "v": 50021, "d": 2048, "entropy": True,
         "weight": False},
        # a training step's gradients at the head of a large model
        {"name": "head_back_2048_tokens", "op": "head_back", "t": 2048, "v": 128256, "d": 4096, "entropy": False,
         "weight": True},
        # the norm of one decoding step, handing 8 bits to the next product
        {"name": "layernorm_1_row_e4m3", "op": "layernorm", "t": 1, "d": 4096, "x": "bf16", "y": "e4m3",
         "residual": True, "bias": True},
        # the norm of a calibration batch, an odd number of rows
        {"name": "layernorm_16381_rows", "op": "layernorm", "t": 16381, "d": 8192, "x": "bf16", "y": "bf16",
         "residual": True, "bias": True},
        # its gradients, few ragged rows in fp32 and many in bf16
        {"name": "layernorm_back_37_rows", "op": "layernorm_back", "t": 37, "d": 11003, "x": "f32", "residual": False},
        {"name": "layernorm_back_8192_rows", "op": "layernorm_back", "t": 8192, "d": 4096, "x": "bf16",
         "residual": True},
        # one token's sample carried back through a 4096 x 4096 projection, 4-bit groups of 128
        {"name": "linear_back_1_token", "op": "linear_back", "t": 1, "m": 4096, "n": 4096, "bits": 4, "group": 128},
        # a few samples through an MLP's down-projection with 8-bit codes, ragged sides
        {"name": "linear_back_17_tokens_8_bits", "op": "linear_back", "t": 17, "m": 4099, "n": 11003, "bits": 8,
         "group": 0},
        # a calibration batch's samples through an MLP's up-projection, 3-bit groups of 128
        {"name": "linear_back_4096_tokens", "op": "linear_back", "t": 4096, "m": 11008, "n": 4096, "bits": 3,
         "group": 128},
    ]


def _between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["head", "head_back", "layernorm", "layernorm_back", "linear_back", "linear_back"])
    if op in ("head", "head_back"):
        v, d = _between(rng, 500, 128256), 8 * _between(rng, 8, 1024)     # hidden sizes are multiples of 8
        case = {"op": op, "t": 0, "v": v, "d": d}
        most = 4095 * 128256 * 4096
        if op == "head_back":
            case["entropy"], case["weight"] = rng.random() < 0.5, rng.random() < 0.5
            most = 2048 * 128256 * 4096
        case["t"] = _between(rng, 1, max(1, min(4096, most // (v * d))))
        return case
    if op == "linear_back":
        bits = rng.choice([2, 3, 4, 4, 8])
        group = rng.choice([0, 0, 32, 64, 128])
        t, m, n = _between(rng, 1, 4096), _between(rng, 128, 28672), _between(rng, 128, 11008)
        if group:
            n = max(1, n // group) * group
        elif rng.random() < 0.5:
            n = n // 128 * 128
        return {"op": op, "t": max(1, min(t, 4096 * 11008 * 4096 // (m * n))), "m": m, "n": n, "bits": bits,
                "group": group}
    d = _between(rng, 64, 16384)
    t = _between(rng, 1, min(16384, (16381 * 8192 if op == "layernorm" else 8192 * 4096) // (2 * d)))
    if rng.random() < 0.5:
        d = max(64, d // 64 * 64)
    case = {"op": op, "t": t, "d": d, "x": rng.choice(["bf16", "f32"]), "residual": rng.random() < 0.5}
    if op == "layernorm":
        case["y"], case["bias"] = rng.choice(["e4m3", case["x"]]), rng.random() < 0.5
    return case


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _hidden(g, t, d):
    """Rows of a residual stream: uneven channels, a few of them large, with offsets."""
    chan = 0.5 + torch.rand(d, generator=g, device="cuda")
    chan[torch.randint(0, d, (max(1, d // 512),), generator=g, device="cuda")] *= 8
    return (torch.randn(t, d, generator=g, device="cuda") + 0.5 * torch.randn(d, generator=g, device="cuda")) * chan


def prepare(case, seed):
    g = _gen(seed)
    s = {"case": case}
    t = case["t"]
    if case["op"] in ("head", "head_back"):
        v, d = case["v"], case["d"]
        s["h"] = torch.randn(t, d, generator=g, device="cuda").bfloat16()       # what the last norm leaves
        s["weight"] = torch.randn(v, d, generator=g, device="cuda", dtype=torch.bfloat16) * (2.5 / d ** 0.5)
        at = torch.randint(0, v, (t,), generator=g, device="cuda")
        at[torch.rand(t, generator=g, device="cuda") < 0.05] = -100             # positions that are not scored
        s["targets"] = at
        if case["op"] == "head_back":
            # the weights of a mean over the scored positions
            s["dlogp"] = -(0.5 + torch.rand(t, generator=g, device="cuda")) / t
            s["dentropy"] = 0.1 * torch.randn(t, generator=g, device="cuda") / t if case["entropy"] else None
            lse, entropy = [], []
            for i in range(0, t, 1024):     # what the forward pass left
                x = s["h"][i:i + 1024].float() @ s["weight"].float().t()
                top = x.amax(1, keepdim=True)
                e = torch.exp(x - top)
                z = e.sum(1)
                lse.append(top[:, 0] + torch.log(z))
                entropy.append(torch.log(z) - (e * (x - top)).sum(1) / z)
            s["lse"], s["entropy"] = torch.cat(lse), torch.cat(entropy)
    elif case["op"] == "linear_back":
        m, n, group = case["m"], case["n"], case["group"]
        qmax, G = 2 ** case["bits"] - 1, (n // group if group else 1)
        s["codes"] = torch.randint(0, qmax + 1, (m, n), generator=g, device="cuda", dtype=torch.uint8)
        s["scales"] = (0.5 + torch.rand(m, G, generator=g, device="cuda")) * (0.08 / qmax)
        s["zeros"] = torch.round((0.4 + 0.2 * torch.rand(m, G, generator=g, device="cuda")) * qmax)
        s["dy"] = _hidden(g, t, m).bfloat16()
        if own:     # a program keeps the weight laid out for its products
            import paper_2608_06291_gb300 as P
            s["packed"] = P.bakron_pack_weight(s["codes"], s["scales"], s["zeros"], qmax, group)
    else:
        d, dt = case["d"], DTYPES[case["x"]]
        s["x"] = _hidden(g, t, d).to(dt)
        s["weight"] = (1 + 0.2 * torch.randn(d, generator=g, device="cuda")).to(dt)
        s["bias"] = (0.1 * torch.randn(d, generator=g, device="cuda")).to(dt) if case.get("bias") else None
        s["residual"] = torch.randn(t, d, generator=g, device="cuda").to(dt) if case["residual"] else None
        if case["op"] == "layernorm_back":     # the residual stream's own gradient joins the norm's
            s["dy"] = torch.randn(t, d, generator=g, device="cuda").to(dt)
    return s


def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    import paper_2608_06291_gb300 as P
    case = s["case"]
    if case["op"] == "head":
        logp, entropy, lse = P.bakron_head_logprobs(s["h"], s["weight"], s["targets"])
        return {"logp": logp, "entropy": entropy, "lse": lse}
    if case["op"] == "head_back":
        dh, dweight = P.bakron_head_logprobs_backward(s["h"], s["weight"], s["targets"], s["lse"], s["dlogp"],
                                                      entropy=s["entropy"], dentropy=s["dentropy"],
                                                      weight_grad=case["weight"])
        return {"dh": dh, "dweight": dweight}
    if case["op"] == "linear_back":
        return P.bakron_linear_backward(s["dy"], s["packed"])
    if case["op"] == "layernorm":
        y, scales, total = P.bakron_layernorm(s["x"], s["weight"], s["bias"], EPS, residual=s["residual"],
                                              out_dtype=DTYPES[case["y"]])
        return {"y": y, "scales": scales, "sum": total}
    dx, dweight, dbias = P.bakron_layernorm_backward(s["dy"], s["x"], s["weight"], EPS, dsum=s["residual"])
    return {"dx": dx, "dweight": dweight, "dbias": dbias}


def _plain(s):
    case = s["case"]
    if case["op"] == "head":
        x, at = s["h"].float() @ s["weight"].float().t(), s["targets"]
        top = x.amax(1, keepdim=True)
        e = torch.exp(x - top)
        z = e.sum(1)
        lse = top[:, 0] + torch.log(z)
        entropy = torch.log(z) - (e * (x - top)).sum(1) / z
        logp = torch.where(at >= 0, x.gather(1, at.clamp(min=0)[:, None])[:, 0] - lse, 0)
        return {"logp": logp, "entropy": entropy, "lse": lse}
    if case["op"] == "head_back":
        h, w, at = s["h"].float(), s["weight"].float(), s["targets"]
        logp = h @ w.t() - s["lse"][:, None]
        p = torch.exp(logp)
        g = torch.where(at >= 0, s["dlogp"], 0)
        d = -g[:, None] * p
        if s["dentropy"] is not None:
            d = d - s["dentropy"][:, None] * p * (logp + s["entropy"][:, None])
        d.scatter_add_(1, at.clamp(min=0)[:, None], g[:, None])
        return {"dh": (d @ w).bfloat16(), "dweight": (d.t() @ h).bfloat16() if case["weight"] else None}
    if case["op"] == "linear_back":
        # the weight is held as codes; its values are formed within the call, as a program does
        # that has no room for both
        m, n = s["codes"].shape
        G = s["scales"].shape[1]
        w = s["codes"].float().view(m, G, n // G)
        w = ((w - s["zeros"][:, :, None]) * s["scales"][:, :, None]).view(m, n)
        return (s["dy"].float() @ w).bfloat16()
    h, w = s["x"].float(), s["weight"].float()
    if case["op"] == "layernorm":
        if s["residual"] is not None:
            h = h + s["residual"].float()
        c = h - h.mean(1, keepdim=True)
        y = c * torch.rsqrt((c * c).mean(1, keepdim=True) + EPS) * w
        if s["bias"] is not None:
            y = y + s["bias"].float()
        scales = None
        if case["y"] == "e4m3":
            scales = y.abs().amax(1) / E4M3_MAX
            scales = torch.where(scales == 0, 1.0, scales)
            y = y / scales[:, None]
        return {"y": y.to(DTYPES[case["y"]]), "scales": scales,
                "sum": h.to(s["x"].dtype) if s["residual"] is not None else None}
    dy = s["dy"].float()
    c = h - h.mean(1, keepdim=True)
    r = torch.rsqrt((c * c).mean(1, keepdim=True) + EPS)
    xhat, back = c * r, dy * w
    dx = r * (back - back.mean(1, keepdim=True) - xhat * (back * xhat).mean(1, keepdim=True))
    if s["residual"] is not None:
        dx = dx + s["residual"].float()
    return {"dx": dx.to(s["x"].dtype), "dweight": (dy * xhat).sum(0), "dbias": dy.sum(0)}


def work(case):
    t = case["t"]
    if case["op"] == "head":
        v, d = case["v"], case["d"]
        return {"bytes": 2 * (v + t) * d + 20 * t, "flops": 2.0 * t * v * d}
    if case["op"] == "head_back":     # the products for p, for dh and, where it is wanted, for dweight
        v, d = case["v"], case["d"]
        both = 2 if case["weight"] else 1
        return {"bytes": 2 * both * v * d + 4 * t * d + t * (16 + (8 if case["entropy"] else 0)),
                "flops": 2.0 * (1 + both) * t * v * d}
    if case["op"] == "linear_back":
        m, n = case["m"], case["n"]
        G = n // case["group"] if case["group"] else 1
        return {"bytes": m * n * (0.5 if case["bits"] <= 4 else 1) + 5 * m * G + 2 * t * (m + n),
                "flops": 2.0 * t * m * n}
    d, size = case["d"], 2 if case["x"] == "bf16" else 4
    if case["op"] == "layernorm":
        out = {"bf16": 2, "f32": 4, "e4m3": 1}[case["y"]]
        scales = 4 * t if case["y"] == "e4m3" else 0
        return {"bytes": t * d * (size * (3 if case["residual"] else 1) + out) + (2 if case["bias"] else 1) * size * d
                + scales, "flops": 8.0 * t * d}
    return {"bytes": t * d * size * (4 if case["residual"] else 3) + (size + 8) * d, "flops": 14.0 * t * d}


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
    t = case["t"]
    if case["op"] == "head":
        h, out = s["h"].double(), {"logp": 0, "entropy": 0, "lse": 0}
        logits = torch.empty(t, case["v"], dtype=torch.float64, device="cuda")
        for i in range(0, case["v"], 8192):
            torch.matmul(h, s["weight"][i:i + 8192].double().t(), out=logits[:, i:i + 8192])
        out["lse"] = torch.logsumexp(logits, 1)
        at = s["targets"]
        picked = torch.take_along_dim(logits, at.clamp(min=0)[:, None], 1)[:, 0] - out["lse"]
        out["logp"] = picked.masked_fill(at < 0, 0.0)
        out["entropy"] = torch.cat([-torch.special.xlogy(p, p).sum(1)
                                    for p in (torch.softmax(part, 1) for part in logits.split(256))])
        return out
    if case["op"] == "head_back":
        h, at = s["h"].double(), s["targets"]
        g = s["dlogp"].double().masked_fill(at < 0, 0.0)
        dh = torch.zeros_like(h)
        dweight = torch.empty(case["v"], case["d"], dtype=torch.float64, device="cuda") if case["weight"] else None
        for i in range(0, case["v"], 8192):
            w = s["weight"][i:i + 8192].double()
            p = (h @ w.t() - s["lse"].double()[:, None]).exp()
            own_token = at[:, None] == torch.arange(i, i + w.shape[0], device="cuda")[None]
            z = g[:, None] * (own_token.double() - p)
            if s["dentropy"] is not None:
                z -= s["dentropy"].double()[:, None] * (torch.special.xlogy(p, p) + p * s["entropy"].double()[:, None])
            dh += z @ w
            if case["weight"]:
                dweight[i:i + 8192] = z.t() @ h
        return {"dh": dh, "dweight": dweight}
    if case["op"] == "linear_back":
        dy = s["dy"].double()
        group = case["group"] or case["n"]
        dx = torch.zeros(t, case["n"], dtype=torch.float64, device="cuda")
        for i in range(0, case["m"], 4096):
            w = s["codes"][i:i + 4096].double()
            w -= s["zeros"][i:i + 4096].double().repeat_interleave(group, 1)
            w *= s["scales"][i:i + 4096].double().repeat_interleave(group, 1)
            dx += dy[:, i:i + 4096] @ w
        return dx
    h = s["x"].double()
    if case["op"] == "layernorm":
        if s["residual"] is not None:
            h = h + s["residual"].double()
        var, mean = torch.var_mean(h, 1, correction=0, keepdim=True)
        y = (h - mean) / torch.sqrt(var + EPS) * s["weight"].double()
        if s["bias"] is not None:
            y += s["bias"].double()
        scales = None
        if case["y"] == "e4m3":
            scales = y.abs().max(1).values / E4M3_MAX
            scales[scales == 0] = 1.0
            y = _round_e4m3(y / scales[:, None])
        return {"y": y, "scales": scales, "sum": h if s["residual"] is not None else None}
    dy = s["dy"].double()
    var, mean = torch.var_mean(h, 1, correction=0, keepdim=True)
    sigma = torch.sqrt(var + EPS)
    xhat = (h - mean) / sigma
    back = dy * s["weight"].double()
    back = back - back.sum(1, keepdim=True) / case["d"]
    dx = (back - xhat * ((back * xhat).sum(1, keepdim=True) / case["d"])) / sigma
    if s["residual"] is not None:
        dx += s["residual"].double()
    return {"dx": dx, "dweight": torch.einsum("td,td->d", dy, xhat), "dbias": torch.ones(t, dtype=torch.float64, device="cuda") @ dy}
