"""Quantise a small residual model with BaKron, run it on its codes and score it.

The model (random weights): an embedding, residual blocks of norm, up-projection with GELU
and down-projection, a last norm and an output head.  What happens:

1. a calibration pass in bf16 keeps every layer's input;
2. ``bakron_token_logprobs`` scores it, its gradient gives samples at the logits, and
   ``bakron_rmsnorm_backward`` carries them to the residual stream, where the last
   down-projection's output is: with them the head and that projection get both Kronecker
   factors, the other layers their input's alone (GPTQ);
3. each weight is rounded, and laid out by ``bakron_pack_weight``;
4. the quantised model runs on the codes: ``bakron_rmsnorm`` hands 8-bit tokens to
   ``bakron_linear``, which adds the residual in its epilogue;
5. both models, and one rounded to nearest, are scored on the same tokens.

    python examples/score_quantized.py
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2608_06291_gb300 as P  # noqa: E402

EPS = 1e-5


def make_model(hidden, wide, vocab, blocks, seed, device="cuda"):
    g = torch.Generator(device=device).manual_seed(seed)

    def w(m, n):
        return (torch.randn(m, n, generator=g, device=device) / n ** 0.5).bfloat16()

    return {"embed": torch.randn(vocab, hidden, generator=g, device=device).bfloat16(),
            "blocks": [{"norm": (1 + 0.1 * torch.randn(hidden, generator=g, device=device)).bfloat16(),
                        "up": w(wide, hidden), "down": w(hidden, wide)} for _ in range(blocks)],
            "norm": torch.ones(hidden, dtype=torch.bfloat16, device=device), "head": 3 * w(vocab, hidden)}


def forward(model, tokens):
    """The bf16 model: (logits, inputs of every layer, the residual stream before the head's norm)."""
    h, inputs = model["embed"][tokens], []
    for b in model["blocks"]:
        x = P.bakron_rmsnorm(h, b["norm"], EPS)[0]
        a = torch.nn.functional.gelu((x @ b["up"].T).float()).bfloat16()
        inputs.append({"up": x, "down": a})
        h = h + a @ b["down"].T
    x = P.bakron_rmsnorm(h, model["norm"], EPS)[0]
    return x @ model["head"].T, inputs, h, x


def quantize(W, a, b, bits, group):
    """Codes, scales, zeros of W from samples of its inputs and (or None) its outputs' gradients."""
    m = W.shape[0]
    A = P.bakron_gram(a, alpha=1.0 / a.shape[0])
    B = P.bakron_gram(b, alpha=1.0 / b.shape[0]) if b is not None else torch.eye(m, device=W.device)
    solve = P.bakron_solve if b is not None else P.bakron_solve_gptq
    return solve(W, P.bakron_prepare(A, B, 0.1), bits, group)


def nearest(W, bits, group):
    """The same grids, every weight rounded on its own."""
    m, n = W.shape
    w = W.float().view(m, n // group, group)
    lo, hi = w.amin(2, keepdim=True).clamp(max=0), w.amax(2, keepdim=True).clamp(min=0)
    s = (hi - lo) / (2 ** bits - 1)
    z = torch.round(-lo / s)
    c = (torch.round(w / s) + z).clamp(0, 2 ** bits - 1)
    return c.to(torch.uint8).view(m, n), s[..., 0].contiguous(), z[..., 0].contiguous()


def packed(layers, bits, group):
    return {k: P.bakron_pack_weight(*v, 2 ** bits - 1, group) for k, v in layers.items()}


def run_quantized(model, weights, tokens):
    """The model on packed codes; returns logits."""
    h, r = model["embed"][tokens], None
    e4m3 = torch.float8_e4m3fn
    for i, b in enumerate(model["blocks"]):
        x, scales, _ = P.bakron_rmsnorm(h, b["norm"], EPS, out_dtype=e4m3)
        a = P.bakron_linear(x, weights[f"up{i}"], x_scales=scales, activation="gelu")
        h = P.bakron_linear(a, weights[f"down{i}"], residual=h)
    x, scales, _ = P.bakron_rmsnorm(h, model["norm"], EPS, out_dtype=e4m3)
    return P.bakron_linear(x, weights["head"], x_scales=scales)


def main(hidden=512, wide=1024, vocab=4000, blocks=2, count=4096, bits=3, group=128, seed=0):
    model = make_model(hidden, wide, vocab, blocks, seed)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    tokens = torch.randint(0, vocab, (count,), generator=g, device="cuda")
    logits, inputs, h, x = forward(model, tokens)
    # what the model itself would say next: the text it is calibrated on
    targets = torch.multinomial(torch.softmax(logits.float(), 1), 1, generator=g)[:, 0]
    logp, entropy, lse, _, best = P.bakron_token_logprobs(logits, targets, top=1)
    # samples at the logits, and from there at the residual stream
    dlogits = P.bakron_token_logprobs_backward(logits, targets, lse, torch.ones_like(logp))
    dh, _ = P.bakron_rmsnorm_backward((dlogits @ model["head"]).contiguous(), h, model["norm"], EPS)

    bakron, plain = {}, {}
    for i, b in enumerate(model["blocks"]):
        last = i == blocks - 1
        for name in ("up", "down"):
            bakron[f"{name}{i}"] = quantize(b[name], inputs[i][name], dh if last and name == "down" else None, bits, group)
            plain[f"{name}{i}"] = nearest(b[name], bits, group)
    bakron["head"], plain["head"] = quantize(model["head"], x, dlogits, bits, group), nearest(model["head"], bits, group)

    out = {"bf16": (logp, entropy, best)}
    for name, layers in (("nearest", plain), ("bakron", bakron)):
        q = run_quantized(model, packed(layers, bits, group), tokens)
        l, e, _, _, ids = P.bakron_token_logprobs(q, targets, top=1)
        out[name] = (l, e, ids)
    report = {k: {"logp": float(l.mean()), "entropy": float(e.mean()), "same best": float((ids == best).float().mean())}
              for k, (l, e, ids) in out.items()}
    for k, v in report.items():
        print(f"{k:8s} mean log probability {v['logp']:8.4f}  entropy {v['entropy']:7.4f}  same best token {v['same best']:.3f}")
    return report


if __name__ == "__main__":
    P.build()
    main()
