"""A small block whose matrices stay in 4 bits, fine-tuned through low-rank adapters, then served to many tenants at once.

    python examples/fp4_adapters.py [--steps 40] [--format e8m0_32]

The block is norm -> up projection -> squared relu -> down projection on a residual stream.  Both projections are stored 4-bit operands; beside each lie the
adapters of several tenants, one for every token, which are all that is trained: in BF16, by an AdamW step with moments in 8 bits.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2512_22804_b200 import adapters, fp4, norm, optim  # noqa: E402


class Block(torch.nn.Module):
    """(x, h) -> (what to add to h, h): h is the residual stream, x what the block before gave."""

    def __init__(self, width: int, hidden: int, tenants: int, rank: int, format: str):
        super().__init__()
        bf16 = dict(device="cuda", dtype=torch.bfloat16)
        self.gain = torch.nn.Parameter(torch.ones(width, **bf16))
        self.up, self.up_t = fp4.quantize(torch.randn(hidden, width, **bf16) * width ** -0.5, format, cols=True)
        self.down, self.down_t = fp4.quantize(torch.randn(width, hidden, **bf16) * hidden ** -0.5, format, cols=True)
        self.a_up = torch.nn.Parameter(torch.randn(tenants, rank, width, **bf16) * width ** -0.5)
        self.b_up = torch.nn.Parameter(torch.zeros(tenants, hidden, rank, **bf16))
        self.a_down = torch.nn.Parameter(torch.randn(tenants, rank, hidden, **bf16) * hidden ** -0.5)
        self.b_down = torch.nn.Parameter(torch.zeros(tenants, width, rank, **bf16))

    def forward(self, x, h, ids):
        y, h = norm.rms_norm(x, self.gain, h)
        y = adapters.linear(y, self.up, self.a_up, self.b_up, ids, 2.0, w_t=self.up_t)
        y = torch.relu(y) ** 2
        return adapters.linear(y, self.down, self.a_down, self.b_down, ids, 2.0, w_t=self.down_t), h


def run(steps=40, format="e8m0_32", tokens=600, width=256, hidden=512, tenants=6, rank=8, seed=0):
    """Losses of the steps, and the largest difference between serving a batch of all tenants at once and token by token."""
    torch.manual_seed(seed)
    block = Block(width, hidden, tenants, rank, format)
    target = torch.randn(tenants + 1, width, device="cuda")                   # one for each tenant; the last for tokens without an adapter
    optimizer = optim.AdamW(block.parameters(), lr=5e-3, bits=8, weight_decay=0.0)
    losses = []
    for _ in range(steps):
        x = torch.randn(tokens, width, device="cuda").to(torch.bfloat16)
        h = torch.randn(tokens, width, device="cuda")
        ids = torch.randint(-1, tenants, (tokens,), device="cuda", dtype=torch.int32)
        out, h = block(x, h, ids)
        loss = ((out.float() - target[ids.long()]) ** 2).mean()
        optimizer.zero_grad()
        loss.backward()
        optimizer.step()
        losses.append(loss.detach())
    fp4.check()
    with torch.no_grad():
        x, h = torch.randn(24, width, device="cuda").to(torch.bfloat16), torch.randn(24, width, device="cuda")
        ids = torch.arange(24, device="cuda", dtype=torch.int32) % (tenants + 1) - 1
        whole = block(x, h, ids)[0].float()
        single = torch.cat([block(x[i:i + 1], h[i:i + 1], ids[i:i + 1])[0] for i in range(24)]).float()
    fp4.check()
    return [float(v) for v in losses], float((whole - single).abs().max()), float(whole.abs().max())


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--steps", type=int, default=40)
    p.add_argument("--format", default="e8m0_32", choices=("e4m3_16", "e8m0_32"))
    a = p.parse_args()
    losses, apart, size = run(a.steps, a.format)
    print("loss %.4f -> %.4f over %d steps" % (losses[0], sum(losses[-5:]) / 5, a.steps))
    print("served token by token: at most %.3g from the batch (values up to %.3g)" % (apart, size))
