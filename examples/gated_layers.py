"""Train a small feed-forward block with a gated projection, then serve it in 8-bit integers.

Training: a layer norm, the gated projection (dense; its input, which is all that it saves, is stored compressed by hooks.SavedActivations), and the
projection behind it in microscaled 4-bit form, whose saved operand is the gated one's output.  Afterwards both projections' weights are stored in 8-bit
integers once, with a scale for each output channel, and tokens are answered one at a time from a graph: norm, quantise, gated
product, quantise, product.

    python examples/gated_layers.py [steps]
"""
from __future__ import annotations

import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

from paper_2510_11400_amd import api, hooks, layers  # noqa: E402


class Model(torch.nn.Module):
    def __init__(self, features: int, hidden: int, classes: int):
        super().__init__()
        kind = dict(device="cuda", dtype=torch.bfloat16)
        self.norm = layers.LayerNorm(features, **kind)
        self.gated = layers.GatedLinear(features, hidden, activation="silu", **kind)
        self.down = torch.nn.Linear(hidden, classes, **kind)
        self.stored = None

    def freeze(self) -> None:
        self.gated.freeze()
        self.stored = api.fh_q8_quantize(self.down.weight.detach())

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        h = self.gated(self.norm(x))
        if self.stored is None:
            return layers.mx_linear(h, self.down.weight, self.down.bias)
        return layers.q8_linear(h, self.stored, self.down.bias)


def main(steps: int = 60, tokens: int = 4096, features: int = 256, hidden: int = 512, classes: int = 16):
    """Returns (the first loss, the last one, the share of tokens that the served model puts in their class)."""
    torch.manual_seed(0)
    model = Model(features, hidden, classes)
    centres = torch.randn(classes, features, device="cuda")
    optimiser = torch.optim.AdamW(model.parameters(), lr=2e-3)
    losses = []
    for step in range(steps):
        label = torch.randint(classes, (tokens,), device="cuda")
        x = (centres[label] + 2.0 * torch.randn(tokens, features, device="cuda")).bfloat16()
        with hooks.SavedActivations(64, 8, exclude=model.parameters(), first_tensor_id=16 * step):
            loss = torch.nn.functional.cross_entropy(model(x).float(), label)
        optimiser.zero_grad()
        loss.backward()
        optimiser.step()
        losses.append(loss.detach())

    model.freeze()
    label = torch.randint(classes, (64,), device="cuda")
    prompt = (centres[label] + 2.0 * torch.randn(64, features, device="cuda")).bfloat16()
    token = prompt[:1].clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side), torch.no_grad():
        model(token)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph), torch.no_grad():
        answer = model(token)
    right = 0
    for i in range(64):
        token.copy_(prompt[i:i + 1])
        graph.replay()
        right += int(answer.argmax()) == int(label[i])
    return float(losses[0]), float(losses[-1]), right / 64


if __name__ == "__main__":
    first, last, share = main(int(sys.argv[1]) if len(sys.argv) > 1 else 60)
    print(f"loss {first:.3f} -> {last:.3f}; served from 8-bit weights, one token at a time: {100 * share:.0f} % right")
