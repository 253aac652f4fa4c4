"""The example of a dense model: its gradients against automatic differentiation in
64 bits, its served step against the 8-bit formula and in a graph."""
import importlib.util
import os

import pytest
import torch

import fused_ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def load():
    spec = importlib.util.spec_from_file_location("dense_step", os.path.join(ROOT, "examples", "dense_step.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.gpu
@pytest.mark.parametrize("tokens", [24, 300])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_gradients(tokens, dtype):
    module = load()
    model = module.Model(hidden=72, inner=50, vocab=611, dtype=dtype)
    g = torch.Generator("cuda").manual_seed(2)
    ids = torch.randint(0, 611, (tokens,), device="cuda", generator=g)
    targets = torch.randint(0, 611, (tokens,), device="cuda", generator=g)
    targets[3] = -1
    loss, gradients = module.loss_and_gradients(model, ids, targets)

    x = model.embedding[ids].double()
    w = {n: getattr(model, n).double().requires_grad_() for n in ("up", "down", "head")}
    gate, lift = (x @ w["up"].t()).chunk(2, 1)
    logits = (x + gate * torch.sigmoid(gate) * lift @ w["down"]) @ w["head"].t()
    lse = torch.logsumexp(logits, 1)
    kept = targets >= 0
    nll = lse - logits.gather(1, targets.clamp(min=0)[:, None])[:, 0]
    exact = (nll + 1e-4 * lse ** 2)[kept].mean()
    exact.backward()
    exact = exact.detach()
    # Everything passed on is rounded to 16 bits: x, inner, hidden, pre, the slopes, their products.  Each
    # rounding moves what follows by at most half a step of it: eight of them on the longest path, of
    # quantities that the path's factors make no larger than the result's own scale; the logits (up to 10
    # in size) move the probabilities by 2 * 10 half steps.
    step = fused_ref.half(dtype)
    assert abs(float(loss) - float(exact)) <= 20 * step * (1 + abs(float(exact)))
    for name, t in gradients.items():
        ref = w[name].grad
        assert t.shape == ref.shape
        assert float((t.double() - ref).norm()) <= 28 * step * float(ref.norm()), name


@pytest.mark.gpu
@pytest.mark.parametrize("tokens", [1, 5, 40])
def test_served_step(tokens):
    module = load()
    model = module.Model(vocab=1003)
    served = module.Served(model, tokens)
    start = torch.arange(tokens, device="cuda")
    served.ids.copy_(start)
    graph = module.record(served)
    eager = []
    served.ids.copy_(start)
    for _ in range(4):
        x = served.embedding[served.ids]
        served.step()
        q, s = fused_ref.scaled_rows(x)
        y, bound = fused_ref.scaled(q.cuda(), served.up, s.cuda(), served.up_scales, torch.float32)
        fused_ref.check(served.both, y, bound, "block")
        eager.append([served.ids.clone(), served.logits.clone()])
    served.ids.copy_(start)
    for ids, logits in eager:
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(served.ids, ids) and torch.equal(served.logits, logits)
