"""A training step of a small dense model, and the same model served in 8-bit
integers, on random weights:

    python examples/dense_step.py [--tokens 512] [--steps 8]

The model is one gated feed-forward block with a residual connection and an output
head.  The training step: the block's inner values (gated) with their
down-projection (gemm), log probabilities of the next tokens straight from the head's
weights (head_logprobs), and back through the head (head_logprobs_grad), the
down-projection (gemm) and the block (gated_grad).  Neither the logits nor their
gradient are ever whole in memory.

Served, its weights are rows of 8-bit integers with a scale for each channel
(scaled_rows); a token's activations become 8-bit on the way into each product
(gemm_scaled), recorded into a graph.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2609_16389_amd import xgemm as xg  # noqa: E402


class Model:
    """Random weights: `embedding` (V, H), `up` (2 I, H), `down` (I, H), `head` (V, H)."""

    def __init__(self, hidden=256, inner=680, vocab=4099, dtype=torch.bfloat16, device="cuda", seed=0):
        make = torch.Generator(device).manual_seed(seed)
        rand = lambda *shape: torch.randn(*shape, device=device, generator=make)  # noqa: E731
        self.embedding = rand(vocab, hidden).to(dtype)
        self.up = (rand(2 * inner, hidden) / hidden ** 0.5).to(dtype)
        self.down = (rand(inner, hidden) / inner ** 0.5).to(dtype)
        self.head = (rand(vocab, hidden) / hidden ** 0.5).to(dtype)


def loss_and_gradients(model, ids, targets, z=1e-4):
    """(loss, gradients of up, down and head) of mean(-logprob) + z * mean(lse^2) over
    the targets that are not negative."""
    x = model.embedding[ids]
    pre = torch.empty(len(ids), len(model.up), dtype=x.dtype, device=x.device)
    inner = xg.gated(x, model.up, pre=pre)
    hidden = (x + xg.gemm(inner, model.down)).to(x.dtype)
    out = xg.head_logprobs(hidden, model.head, targets)

    kept = (targets >= 0).float()
    weight = kept / kept.sum().clamp(min=1)
    loss = (weight * (z * out["lse"] ** 2 - out["logprob"])).sum()

    d_hidden, d_head = xg.head_logprobs_grad(hidden, model.head, targets, out["lse"], -weight, 2 * z * weight * out["lse"])
    d_down = xg.gemm(inner.t().contiguous(), d_hidden)
    d_inner = xg.gemm(d_hidden, model.down.t().contiguous()).to(x.dtype)
    _, d_up = xg.gated_grad(x, model.up, pre, d_inner, out=(None, torch.empty_like(model.up)))
    return loss, {"up": d_up, "down": d_down, "head": d_head}


class Served:
    """The model in 8-bit integers, with the buffers of a step for `tokens` sequences."""

    def __init__(self, model, tokens=1, alternatives=3):
        self.embedding, self.alternatives = model.embedding, alternatives
        self.up, self.up_scales = xg.scaled_rows(model.up)
        self.down, self.down_scales = xg.scaled_rows(model.down.t().contiguous())
        self.head, self.head_scales = xg.scaled_rows(model.head)
        device, dtype = model.head.device, model.head.dtype
        self.ids = torch.zeros(tokens, dtype=torch.int64, device=device)
        self.both = torch.empty(tokens, len(self.up), device=device)
        self.added = torch.empty(tokens, len(self.down), dtype=dtype, device=device)
        self.logits = torch.empty(tokens, len(self.head), device=device)
        self.result = {"top_logprob": torch.empty(tokens, alternatives, device=device),
                       "top_id": torch.empty(tokens, alternatives, dtype=torch.int64, device=device)}

    def step(self):
        """From the tokens in `ids` to the next ones, which take their place."""
        x = self.embedding[self.ids]
        gate, lift = xg.gemm_scaled(x, self.up, self.up_scales, out=self.both).chunk(2, 1)
        inner = torch.nn.functional.silu(gate) * lift
        hidden = x + xg.gemm_scaled(inner, self.down, self.down_scales, out=self.added)
        xg.gemm_scaled(hidden, self.head, self.head_scales, out=self.logits)
        xg.logprobs(self.logits, top=self.alternatives, out=self.result)
        self.ids.copy_(self.result["top_id"][:, 0])


def record(served):
    """A graph of a step, after steps that let the library allocate its workspaces."""
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    ids = served.ids.clone()
    with torch.cuda.stream(stream):
        for _ in range(2):
            served.step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            served.step()
    torch.cuda.current_stream().wait_stream(stream)
    served.ids.copy_(ids)
    return graph


def main(argv=None):
    parser = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    parser.add_argument("--tokens", type=int, default=512, help="tokens of a training step")
    parser.add_argument("--steps", type=int, default=8, help="training steps, and tokens served")
    args = parser.parse_args(argv)

    model = Model()
    make = torch.Generator("cuda").manual_seed(1)
    ids = torch.randint(0, len(model.head), (args.tokens,), device="cuda", generator=make)
    targets = ids.roll(-1)
    targets[-1] = -1
    for k in range(args.steps):
        loss, gradients = loss_and_gradients(model, ids, targets)
        for name, g in gradients.items():
            weight = getattr(model, name)
            weight.copy_(weight.float() - 2.0 * g.float())
        print("step %d: loss %.4f" % (k, float(loss)))

    served = Served(model)
    served.ids.copy_(ids[:1])
    graph = record(served)
    for _ in range(args.steps):
        graph.replay()
        print("token %d, log probability %.2f" % (int(served.ids), float(served.result["top_logprob"][0, 0])))


if __name__ == "__main__":
    main()
