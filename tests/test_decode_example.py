"""The decoding example: its quantiser, its step in a graph against the same
step without one, each of its operators from that operator's own inputs, and the
gradient of the head."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import decode_ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def load():
    spec = importlib.util.spec_from_file_location("decode_step", os.path.join(ROOT, "examples", "decode_step.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_quantiser_rounds_within_a_step():
    w = torch.randn(24, 256, generator=torch.Generator().manual_seed(3))
    q, scales, zeros = load().quantize(w)
    assert q.shape == (24, 128) and scales.shape == zeros.shape == (24, 4)
    k = np.arange(256) // 64
    s = scales.numpy().astype(np.float64)[:, k]
    v = (decode_ref.unpack(q.numpy(), 256) - zeros.numpy().astype(np.float64)[:, k]) * s
    # half a step for the value, and half a step more where the rounded zero
    # point leaves an end of the range uncovered
    assert np.all(np.abs(v - w.numpy()) <= 1.001 * s)


@pytest.mark.gpu
def test_graph_replays_the_step():
    module = load()
    model = module.Model(tokens=3, vocab=4099)
    graph = module.record(model)
    start = model.ids.clone()
    eager = []
    for _ in range(4):
        model.step()
        eager.append([model.ids.clone(), model.logits.clone(), {k: v.clone() for k, v in model.result.items()}])
    model.ids.copy_(start)
    for ids, logits, result in eager:
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(model.ids, ids) and torch.equal(model.logits, logits)
        for name, t in result.items():
            assert torch.equal(model.result[name], t), name


@pytest.mark.gpu
def test_step_against_64_bits():
    model = load().Model(tokens=5)
    before = model.ids.clone()
    model.step()
    torch.cuda.synchronize()
    num = lambda t: t.double().cpu().numpy()  # noqa: E731
    x = num(model.embedding[before])
    y, S = decode_ref.quant(x, model.q.cpu().numpy(), num(model.scales), model.zeros.cpu().numpy(), 64, 512)
    # rounded to bfloat16, after at most 512 + 16 additions of products in fp32
    assert np.all(np.abs(num(model.projected) - y) <= 2.0 ** -8 * np.abs(y) + 528 * 2.0 ** -24 * S)
    x = num(model.embedding[before] + model.projected)
    y, S, ids = decode_ref.experts(x, num(model.scores), num(model.up), num(model.down), 2, True)
    # the same for two products in a row, with h in two parts of 8 bits
    assert np.all(np.abs(num(model.mixed) - y) <= 2.0 ** -8 * np.abs(y) + (2.0 ** -15 + 1024 * 2.0 ** -24) * S)
    logits = num(model.logits)
    ref = decode_ref.logprobs(logits, np.full(5, -1), 5)
    names = ["lse", "logprob", "entropy", "top_logprob", "top_id"]
    ref = dict(zip(names, ref))
    for name in ("lse", "entropy", "top_logprob"):
        assert np.all(np.abs(num(model.result[name]) - ref[name]) <= 1e-5 * (1 + np.abs(ref[name]))), name
    assert np.array_equal(model.result["top_id"].cpu().numpy(), ref["top_id"])
    assert torch.equal(model.ids, model.result["top_id"][:, 0])


@pytest.mark.gpu
def test_gradient_of_the_head():
    module = load()
    g = torch.Generator("cuda").manual_seed(11)
    hidden = torch.randn(24, 64, device="cuda", generator=g).to(torch.bfloat16)
    head = (torch.randn(64, 1000, device="cuda", generator=g) / 8).to(torch.bfloat16)
    targets = torch.randint(0, 1000, (24,), device="cuda", generator=g)
    targets[3] = -1
    loss, gradient = module.head_loss(hidden, head, targets)
    # the formula in 64 bits by automatic differentiation
    h, w = hidden.double().cpu(), head.double().cpu().requires_grad_()
    p = torch.log_softmax(h @ w, 1)
    kept = (targets >= 0).cpu()
    nll = -p[torch.arange(24), targets.cpu().clamp(min=0)][kept].mean()
    exact = nll - 0.01 * (-(p.exp() * p).sum(1)[kept].mean())
    exact.backward()
    exact = exact.detach()
    assert abs(float(loss) - float(exact)) <= 1e-4 * abs(float(exact))
    # the logits' gradient is rounded to bfloat16: half of 2^-8 of each term, so
    # 2^-9 of the sum of their absolute values, and as much again for fp32
    logits = (h @ w.detach()).requires_grad_()
    q = torch.log_softmax(logits, 1)
    (-q[torch.arange(24), targets.cpu().clamp(min=0)][kept].mean() + 0.01 * (q.exp() * q).sum(1)[kept].mean()).backward()
    bound = h.abs().t() @ logits.grad.abs()
    assert torch.all((gradient.double().cpu() - w.grad).abs() <= 2.0 ** -8 * bound + 1e-9)
