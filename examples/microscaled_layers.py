"""Train a small model whose linear layers work in microscaled 4-bit form, then serve it.

Forward and backward run on fh_layer_norm_mx, fh_mx_quantize, fh_mx_matmul and fh_layer_norm_backward; what autograd saves beside
the 4-bit operands (the norms' inputs) is stored compressed by hooks.SavedActivations.  Afterwards the weights are stored in 4 bits
once, and tokens are answered one at a time, two kernels a layer, captured in a graph.

    python examples/microscaled_layers.py [steps]
"""
from __future__ import annotations

import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

from paper_2510_11400_amd import hooks, layers  # noqa: E402


class Model(torch.nn.Module):
    def __init__(self, features: int, hidden: int, classes: int):
        super().__init__()
        kind = dict(rounding="stochastic", device="cuda", dtype=torch.bfloat16)
        self.up = layers.LayerNormMxLinear(features, hidden, tensor_id=0, **kind)
        self.down = layers.LayerNormMxLinear(hidden, classes, tensor_id=1, **kind)

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        return self.down(torch.nn.functional.gelu(self.up(x)))


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

    model.up.freeze()
    model.down.freeze()
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
    print(f"loss {first:.3f} -> {last:.3f}; served from 4-bit weights, one token at a time: {100 * share:.0f} % right")
