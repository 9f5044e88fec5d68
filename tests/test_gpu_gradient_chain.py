"""The gradients together, as samples are carried back through a quantised model: head, layer norm,
product, against the 64-bit formulas; a captured run; the example.

Each step's bf16 result has 2^-8, and its inputs' roundings before it: along a chain of k results, each a
sum of many terms with independent roundings, the norm of the error stays below k (2^-8 + 2^-8) of the
result's norm (a result's own rounding, and its operands').  The head's probabilities also have the
logits' error as a relative one: logits of spread 3 from rounded hidden states, 3 2^-8 / sqrt(3): one step more."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2608_06291_gb300 as P

EX = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "carry_samples.py")


def _example():
    spec = importlib.util.spec_from_file_location("carry_samples", EX)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _setup(count, group):
    m = _example()
    model = m.make_model(256, 384, 1000, 1, 3)
    g = torch.Generator(device="cuda").manual_seed(5)
    tokens = torch.randint(0, 1000, (count,), generator=g, device="cuda")
    targets = torch.randint(0, 1000, (count,), generator=g, device="cuda")
    targets[::7] = -100
    b = model["blocks"][0]
    codes = {k: m.nearest(b[k], 4, group) for k in ("up", "down")}
    packed = {k: P.bakron_pack_weight(*v, 15, group) for k, v in codes.items()}
    values = {k: P.dequantize(*v).double() for k, v in codes.items()}
    return m, model, tokens, targets, packed, values


@pytest.mark.parametrize("count", [1, 13, 600])
@pytest.mark.parametrize("group", [32, 128])
def test_chain(count, group):
    m, model, tokens, targets, packed, values = _setup(count, group)
    b = model["blocks"][0]
    x, h, kept = m.forward(model, tokens, lambda v, i, k: P.bakron_linear(v, packed[k]))
    dx, _ = m.samples_at_stream(model, x, h, targets)
    du, dstream = m.carry(b, kept[0], lambda name, s: packed[name], dx)

    # the same from the calibration's own values, in 64 bits
    def norm(v, wb):
        c = v - v.mean(1, keepdim=True)
        return c / torch.sqrt(c.square().mean(1, keepdim=True) + m.EPS) * wb[0].double() + wb[1].double()

    ok = (targets >= 0).double()

    def score(stream):
        lp = torch.log_softmax(norm(stream, model["norm"]) @ model["head"].double().T, 1)
        return (ok * lp.gather(1, targets.clamp(min=0)[:, None])[:, 0]).sum()

    stream = h.double().requires_grad_()
    want = torch.autograd.grad(score(stream), stream)[0]
    assert torch.linalg.norm(dx.double() - want) <= 3 * 2 * 2.0 ** -8 * torch.linalg.norm(want)
    u = kept[0]["u"].double().requires_grad_()
    a = torch.nn.functional.gelu(u)
    want_u = torch.autograd.grad((a @ values["down"].T * dx.double()).sum(), u)[0]
    assert torch.linalg.norm(du.double() - want_u) <= 2 * 2 * 2.0 ** -8 * torch.linalg.norm(want_u)
    h0 = kept[0]["h"].double().requires_grad_()
    n = norm(h0, b["norm"])
    want_h = torch.autograd.grad((n @ values["up"].T * du.double()).sum(), h0)[0] + dx.double()
    assert torch.linalg.norm(dstream.double() - want_h) <= 2 * 2 * 2.0 ** -8 * torch.linalg.norm(want_h)


def test_captured_beside_an_eager_run():
    """The whole way back in a graph, replayed on new samples while eager results are alive."""
    m, model, tokens, targets, packed, _ = _setup(40, 128)
    b = model["blocks"][0]

    def way(t):
        x, h, kept = m.forward(model, t, lambda v, i, k: P.bakron_linear(v, packed[k]))
        dx, logp = m.samples_at_stream(model, x, h, targets)
        return (logp, dx) + m.carry(b, kept[0], lambda name, s: packed[name], dx)

    eager = way(tokens)
    static = tokens.clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        way(static)
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = way(static)
    other = tokens.flip(0)
    for t in (other, tokens):
        static.copy_(t)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(out, way(t)))
    assert all(torch.equal(a, c) for a, c in zip(out, eager))


def test_example_runs():
    report = _example().main(hidden=256, wide=384, vocab=700, blocks=2, count=1024, bits=4, group=128)
    assert set(report) == {"bf16", "nearest", "bakron"} and all(torch.isfinite(torch.tensor(v)) for v in report.values())
