"""The example that quantises a small model, runs it on its codes and scores it."""
import importlib.util
import math
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_score_quantized():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    spec = importlib.util.spec_from_file_location("score_quantized", os.path.join(ROOT, "examples", "score_quantized.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    example.P.build()
    r = example.main(hidden=256, wide=512, vocab=1000, blocks=2, count=2048, bits=4, group=128)
    assert all(math.isfinite(x) for v in r.values() for x in v.values())
    assert r["bf16"]["same best"] == 1.0
    # rounded under its Hessians the model says more nearly what it said before
    loss = {k: r["bf16"]["logp"] - v["logp"] for k, v in r.items()}
    assert loss["bakron"] < loss["nearest"]


def test_the_operators_follow_the_dense_model():
    """The quantised model on its codes against the same layers dequantised, in torch."""
    spec = importlib.util.spec_from_file_location("score_quantized", os.path.join(ROOT, "examples", "score_quantized.py"))
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    P = ex.P
    model = ex.make_model(256, 512, 1000, 2, 3)
    tokens = torch.randint(0, 1000, (300,), generator=torch.Generator().manual_seed(1)).cuda()
    layers = {f"{n}{i}": ex.nearest(b[n], 4, 128) for i, b in enumerate(model["blocks"]) for n in ("up", "down")}
    layers["head"] = ex.nearest(model["head"], 4, 128)
    got = ex.run_quantized(model, ex.packed(layers, 4, 128), tokens).double()
    h = model["embed"][tokens].double()

    def norm(h, w):
        return h / torch.sqrt(h.square().mean(1, keepdim=True) + ex.EPS) * w.double()

    for i, b in enumerate(model["blocks"]):
        x = norm(h, b["norm"])
        a = torch.nn.functional.gelu(x @ P.dequantize(*layers[f"up{i}"]).double().T)
        h = h + a @ P.dequantize(*layers[f"down{i}"]).double().T
    want = norm(h, model["norm"]) @ P.dequantize(*layers["head"]).double().T
    # three roundings of tokens to e4m3 (2^-4 each, independent over 256 columns) and bf16 between
    assert torch.linalg.norm(got - want) <= 0.06 * torch.linalg.norm(want)
