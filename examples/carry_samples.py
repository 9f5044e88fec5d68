"""Both Kronecker factors for every layer of a small model, from the last layer to the first.

A layer's output-side factor needs samples of the loss's gradient at its output.  They start at the
head and go backward through the layers behind, which by then are quantised:

1. a calibration pass in bf16 keeps what the gradients need, and ``bakron_head_logprobs`` scores
   it without forming logits;
2. ``bakron_head_logprobs_backward`` gives the samples at the last hidden states,
   ``bakron_layernorm_backward`` at the residual stream;
3. block by block, last first: the down-projection is rounded with the samples at its output and laid
   out by ``bakron_pack_weight``; ``bakron_linear_backward`` carries them through the codes and the
   activation's derivative to the up-projection, which is rounded with them; from there through its codes and
   the block's norm, where the gradient of the residual stream joins, to the block before;
4. the quantised model, and one rounded to nearest, are scored on the same tokens.

    python examples/carry_samples.py
"""
from __future__ import annotations

import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2608_06291_gb300 as P  # noqa: E402
from score_quantized import nearest, quantize  # noqa: E402

EPS = 1e-5


def make_model(hidden, wide, vocab, blocks, seed, device="cuda"):
    g = torch.Generator(device=device).manual_seed(seed)

    def w(m, n):
        return (torch.randn(m, n, generator=g, device=device) / n ** 0.5).bfloat16()

    def norm():
        return ((1 + 0.1 * torch.randn(hidden, generator=g, device=device)).bfloat16(),
                (0.1 * torch.randn(hidden, generator=g, device=device)).bfloat16())

    return {"embed": torch.randn(vocab, hidden, generator=g, device=device).bfloat16(),
            "blocks": [{"norm": norm(), "up": w(wide, hidden), "down": w(hidden, wide)} for _ in range(blocks)],
            "norm": norm(), "head": 3 * w(vocab, hidden)}


def forward(model, tokens, product):
    """The hidden states before the head, and what the gradients need; product(x, block, name)."""
    h, kept = model["embed"][tokens], []
    for i, b in enumerate(model["blocks"]):
        x, _, _ = P.bakron_layernorm(h, *b["norm"], EPS)
        u = product(x, i, "up")
        a = torch.nn.functional.gelu(u.float()).bfloat16()
        kept.append({"h": h, "up": x, "u": u, "down": a})
        h = h + product(a, i, "down")
    x, _, _ = P.bakron_layernorm(h, *model["norm"], EPS)
    return x, h, kept


def gelu_back(da, u):
    """da gelu'(u)."""
    u = u.float()
    slope = 0.5 * (1 + torch.erf(u / math.sqrt(2))) + u * torch.exp(-0.5 * u * u) / math.sqrt(2 * math.pi)
    return (da.float() * slope).bfloat16()


def samples_at_stream(model, x, h, targets):
    """Gradients of the tokens' log probabilities at the residual stream before the last norm."""
    logp, _, lse = P.bakron_head_logprobs(x, model["head"], targets)
    dx, _ = P.bakron_head_logprobs_backward(x, model["head"], targets, lse, torch.ones_like(logp), weight_grad=False)
    return P.bakron_layernorm_backward(dx, h, model["norm"][0], EPS)[0], logp


def carry(block, kept, weight, dx):
    """Samples at a block's output -> (at its up-projection's output, at its input), through its codes:
    weight(name) gives the packed weight once its samples are known."""
    du = gelu_back(P.bakron_linear_backward(dx, weight("down", dx)), kept["u"])
    dn = P.bakron_linear_backward(du, weight("up", du))
    return du, P.bakron_layernorm_backward(dn, kept["h"], block["norm"][0], EPS, dsum=dx)[0]


def main(hidden=512, wide=1024, vocab=4000, blocks=2, count=4096, bits=3, group=128, seed=0):
    model = make_model(hidden, wide, vocab, blocks, seed)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    tokens = torch.randint(0, vocab, (count,), generator=g, device="cuda")
    targets = torch.randint(0, vocab, (count,), generator=g, device="cuda")
    qmax = 2 ** bits - 1

    def plain(x, i, name):
        return x @ model["blocks"][i][name].T

    x, h, kept = forward(model, tokens, plain)
    dx, logp = samples_at_stream(model, x, h, targets)
    packed, rounded = {}, {}
    for i in reversed(range(blocks)):
        b = model["blocks"][i]

        def weight(name, samples):
            packed[i, name] = P.bakron_pack_weight(*quantize(b[name], kept[i][name], samples, bits, group), qmax, group)
            rounded[i, name] = P.bakron_pack_weight(*nearest(b[name], bits, group), qmax, group)
            return packed[i, name]

        _, dx = carry(b, kept[i], weight, dx)

    report = {"bf16": float(logp.mean())}
    for name, layers in (("nearest", rounded), ("bakron", packed)):
        x, _, _ = forward(model, tokens, lambda v, i, k: P.bakron_linear(v, layers[i, k]))
        report[name] = float(P.bakron_head_logprobs(x, model["head"], targets)[0].mean())
    for k, v in report.items():
        print(f"{k:8s} mean log probability {v:8.4f}")
    return report


if __name__ == "__main__":
    P.build()
    main()
