"""A decoding step of a small language model, and a training step of its head,
on random weights:

    python examples/decode_step.py [--tokens 4] [--steps 16]

One step takes the embeddings of a few sequences' last tokens through a
projection with 4-bit weights (gemv_quant), a router (gemm) with a
mixture-of-experts layer (experts) and the output head (gemm) to log
probabilities with their most likely alternatives (logprobs).  The step is
recorded into a graph once and replayed for every token.

The tokens generated are then the targets of one step of gradient descent on
the head: loss = -mean(logprob) - bonus * mean(entropy), its gradient in the
logits by logprobs_grad, in the head by gemm.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2609_16389_amd import xgemm as xg  # noqa: E402

GROUP = 64


def quantize(w, group=GROUP):
    """(q, scales, zeros) of a matrix (N, K), K a multiple of the group: 16
    levels between each group's smallest and largest value (or zero)."""
    N, K = w.shape
    g = w.float().view(N, K // group, group)
    low, high = g.amin(2).clamp(max=0), g.amax(2).clamp(min=0)
    scales = ((high - low) / 15).clamp(min=1e-8).to(w.dtype)
    zeros = (-low / scales.float()).round().clamp(0, 15)
    q = (g / scales.float()[..., None] + zeros[..., None]).round().clamp(0, 15).to(torch.uint8).view(N, K)
    return q[:, 0::2] | q[:, 1::2] << 4, scales, zeros.to(torch.uint8)


class Model:
    """Random weights and the buffers of a step for `tokens` sequences."""

    def __init__(self, tokens=4, hidden=512, inner=256, experts=16, top=2, vocab=8192, alternatives=5, dtype=torch.bfloat16,
                 device="cuda", seed=0):
        make = torch.Generator(device).manual_seed(seed)
        rand = lambda *shape: torch.randn(*shape, device=device, generator=make)  # noqa: E731
        self.top, self.alternatives = top, alternatives
        self.embedding = rand(vocab, hidden).to(dtype)
        self.q, self.scales, self.zeros = quantize((rand(hidden, hidden) / hidden ** 0.5).to(dtype))
        self.router = (rand(hidden, experts) / hidden ** 0.5).to(dtype)
        self.up = (rand(experts, 2 * inner, hidden) / hidden ** 0.5).to(dtype)
        self.down = (rand(experts, hidden, inner) / inner ** 0.5).to(dtype)
        self.head = (rand(hidden, vocab) / hidden ** 0.5).to(dtype)

        new = lambda *shape, dtype=dtype: torch.empty(*shape, dtype=dtype, device=device)  # noqa: E731
        self.ids = torch.arange(tokens, device=device)
        self.projected, self.mixed = new(tokens, hidden), new(tokens, hidden)
        self.scores, self.logits = new(tokens, experts, dtype=torch.float32), new(tokens, vocab, dtype=torch.float32)
        self.hidden = new(tokens, hidden)
        self.result = {"lse": new(tokens, dtype=torch.float32), "entropy": new(tokens, dtype=torch.float32),
                       "top_logprob": new(tokens, alternatives, dtype=torch.float32),
                       "top_id": new(tokens, alternatives, dtype=torch.int64)}

    def step(self):
        """From the tokens in `ids` to the next ones, which take their place."""
        x = self.embedding[self.ids]
        x = x + xg.gemv_quant(x, self.q, self.scales, self.zeros, GROUP, out=self.projected)
        xg.gemm(x, self.router, out=self.scores)
        x = x + xg.experts(x, self.scores, self.up, self.down, self.top, out=self.mixed)
        self.hidden.copy_(x)
        xg.gemm(x, self.head, out=self.logits)
        xg.logprobs(self.logits, top=self.alternatives, out=self.result)
        self.ids.copy_(self.result["top_id"][:, 0])


def record(model):
    """A graph of a step, after steps that let the library allocate its workspaces."""
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    ids = model.ids.clone()
    with torch.cuda.stream(stream):
        for _ in range(2):
            model.step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            model.step()
    torch.cuda.current_stream().wait_stream(stream)
    model.ids.copy_(ids)
    return graph


def head_loss(hidden, head, targets, bonus=0.01):
    """(loss, its gradient in the head) for hidden states (R, H), a head (H, V)
    and targets (R,), negative ones left out."""
    logits = xg.gemm(hidden, head)
    out = xg.logprobs(logits, targets)
    count = (targets >= 0).sum().clamp(min=1)
    counted = (targets >= 0).float() / count
    loss = -(out["logprob"] * counted).sum() - bonus * (out["entropy"] * counted).sum()
    # (over the logits, which nothing needs any more)
    xg.logprobs_grad(logits, targets, out["lse"], out["entropy"], d_logprob=-counted, d_entropy=-bonus * counted, out=logits)
    return loss, xg.gemm(hidden.t().contiguous(), logits.to(head.dtype))


def main(argv=None):
    parser = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    parser.add_argument("--tokens", type=int, default=4, help="sequences decoded together")
    parser.add_argument("--steps", type=int, default=16)
    args = parser.parse_args(argv)

    model = Model(args.tokens)
    graph = record(model)
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    hidden, made, likely = [], [], []
    graph_time = 0.0
    for _ in range(args.steps):
        begin.record()
        graph.replay()
        end.record()
        end.synchronize()
        graph_time += begin.elapsed_time(end)
        hidden.append(model.hidden.clone())
        made.append(model.ids.clone())
        likely.append(model.result["top_logprob"][:, 0].clone())
    print("%d steps of %d sequences, %.1f us a step" % (args.steps, args.tokens, 1e3 * graph_time / args.steps))
    for s in range(args.tokens):
        print("sequence %d:" % s, " ".join("%d (%.2f)" % (int(t[s]), float(p[s])) for t, p in zip(made[:8], likely)))

    hidden, targets = torch.cat(hidden), torch.cat(made)
    before, gradient = head_loss(hidden, model.head, targets)
    after, _ = head_loss(hidden, (model.head.float() - 1e-3 * gradient).to(model.head.dtype), targets)
    print("loss of the head %.4f, after a step of 0.001 down its gradient %.4f" % (float(before), float(after)))


if __name__ == "__main__":
    main()
