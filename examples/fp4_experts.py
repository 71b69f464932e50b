"""A small mixture of experts whose matrices are 4-bit: trained for a few steps, then served token by token.

    python examples/fp4_experts.py [--steps 60] [--format e4m3_16]

Each block is a 4-bit linear layer, a router that picks `top` of the experts for every token, and the experts' 4-bit
matrices.  Training quantises activations, weights and gradients along the reduction axis of each of the three products and
passes the rounding straight through; serving quantises the weights once and keeps only their codes and scales.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2512_22804_b200 import experts, fp4  # noqa: E402


class Block(torch.nn.Module):
    """y = experts(relu(x w_in^T)): [tokens, width] -> [tokens, width]."""

    def __init__(self, width: int, hidden: int, n_experts: int, top: int, format: str):
        super().__init__()
        bf16 = dict(device="cuda", dtype=torch.bfloat16)
        self.w_in = torch.nn.Parameter(torch.randn(hidden, width, **bf16) * width ** -0.5)
        self.w_out = torch.nn.Parameter(torch.randn(n_experts, width, hidden, **bf16) * (2 / hidden) ** 0.5)
        self.router = torch.nn.Parameter(torch.randn(n_experts, width, device="cuda") * width ** -0.5)
        self.top, self.format = top, format
        self.stored = None

    def route(self, x):
        weight, ids = torch.topk(torch.softmax(x.float() @ self.router.t(), dim=1), self.top, dim=1)
        return ids.to(torch.int32), weight

    def forward(self, x):
        ids, weight = self.route(x)
        if self.stored is not None:
            a, _ = fp4.quantize(x, self.format)
            return experts.linear(torch.relu(fp4.matmul(a, self.stored[0])), self.stored[1], ids, weight)
        return experts.linear(torch.relu(fp4.linear(x, self.w_in, self.format)), self.w_out, ids, weight, self.format)

    def store(self):
        """Quantises the weights once for serving."""
        self.stored = [fp4.quantize(w.detach(), self.format)[0] for w in (self.w_in, self.w_out)]


def run(steps=60, format="e4m3_16", tokens=512, width=256, hidden=512, n_experts=8, top=2, seed=0):
    """Losses of the steps, and the largest difference between serving a batch at once and token by token."""
    torch.manual_seed(seed)
    block = Block(width, hidden, n_experts, top, format)
    target = torch.randn(width, width, device="cuda") * width ** -0.5
    optimizer = torch.optim.Adam(block.parameters(), lr=2e-3)
    losses = []
    for _ in range(steps):
        x = torch.randn(tokens, width, device="cuda").to(torch.bfloat16)
        loss = ((block(x).float() - torch.tanh(x.float() @ target)) ** 2).mean()
        optimizer.zero_grad()
        loss.backward()
        optimizer.step()
        losses.append(loss.detach())
    fp4.check()
    block.store()
    with torch.no_grad():
        x = torch.randn(16, width, device="cuda").to(torch.bfloat16)
        whole = block(x).float()
        single = torch.cat([block(x[i:i + 1]) for i in range(16)]).float()
    fp4.check()
    return [float(v) for v in losses], float((whole - single).abs().max()), float(whole.abs().max())


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--steps", type=int, default=60)
    p.add_argument("--format", default="e4m3_16", choices=("e4m3_16", "e8m0_32"))
    a = p.parse_args()
    losses, apart, size = run(a.steps, a.format)
    print("loss %.4f -> %.4f over %d steps" % (losses[0], sum(losses[-5:]) / 5, a.steps))
    print("served token by token: at most %.3g from the batch (values up to %.3g)" % (apart, size))
