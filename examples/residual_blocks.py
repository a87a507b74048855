"""A stack of residual blocks trained by K simulated workers with coded gradients: layer norm with the sum of the residual stream,
backward into the workers' flat gradients, encode, decode and average, clipping, AdamW.

    python examples/residual_blocks.py [--steps 100] [--state-bits 8] [--dtype bfloat16]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_1908_06077_amd as nuq  # noqa: E402
from paper_1908_06077_amd.norm import LayerNorm  # noqa: E402
from paper_1908_06077_amd.optim import NUQAdamW  # noqa: E402


class Blocks(torch.nn.Module):
    """stream <- stream + MLP(norm(stream)), `depth` times, then a norm and a linear read-out.  dtype: of the rows and products;
    the parameters are fp32."""

    def __init__(self, width: int, depth: int, out: int, dtype: torch.dtype = torch.float32):
        super().__init__()
        self.dtype = dtype
        self.norms = torch.nn.ModuleList(LayerNorm(width) for _ in range(depth + 1))
        self.up = torch.nn.ModuleList(torch.nn.Linear(width, 4 * width) for _ in range(depth))
        self.down = torch.nn.ModuleList(torch.nn.Linear(4 * width, width) for _ in range(depth))
        self.head = torch.nn.Linear(width, out)

    def _linear(self, layer, x):
        return torch.nn.functional.linear(x, layer.weight.to(x.dtype), layer.bias.to(x.dtype))

    def forward(self, x):
        stream = x.to(self.dtype)
        y = self.norms[0](stream)
        for up, down, norm in zip(self.up, self.down, self.norms[1:]):
            branch = self._linear(down, torch.nn.functional.gelu(self._linear(up, y)))
            y, stream = norm(branch, stream)
        return self._linear(self.head, y).float()


def groups(model, decay=0.1):
    """Weight decay for matrices alone."""
    params = list(model.parameters())
    return [{"params": [p for p in params if p.dim() > 1], "weight_decay": decay},
            {"params": [p for p in params if p.dim() <= 1], "weight_decay": 0.0}]


def train(steps=100, K=4, width=96, depth=2, batch=64, state_bits=32, dtype=torch.float32, lr=2e-3, seed=3):
    """(losses, optimizer) of `steps` steps on a synthetic regression."""
    dev = torch.device("cuda")
    torch.manual_seed(seed)
    model = Blocks(width, depth, 8, dtype).to(dev)
    opt = NUQAdamW(groups(model), K=K, lr=lr, betas=(0.9, 0.95), bucket=512, s=4, max_norm=1.0, state_bits=state_bits, seed=seed)
    g = torch.Generator(device=dev).manual_seed(seed)
    teacher = torch.randn(width, 8, generator=g, device=dev) / width ** 0.5
    losses = []
    for _ in range(steps):
        step = []
        for k in range(K):
            x = torch.randn(batch, width, generator=g, device=dev)
            with opt.worker(k):
                loss = torch.nn.functional.mse_loss(model(x), torch.tanh(2.0 * x @ teacher))
                loss.backward()
            step.append(loss.detach())
        opt.step()
        losses.append(torch.stack(step).mean())
    return torch.stack(losses).tolist(), opt


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=100)
    ap.add_argument("--state-bits", type=int, default=32, choices=(8, 32))
    ap.add_argument("--dtype", default="float32", choices=("float32", "bfloat16", "float16"))
    a = ap.parse_args()
    losses, opt = train(a.steps, state_bits=a.state_bits, dtype=getattr(torch, a.dtype))
    for t in range(0, len(losses), max(1, len(losses) // 10)):
        print("step %4d  loss %.4f" % (t, losses[t]))
    print("last       loss %.4f, norm of the last average %.4f, flags %d" % (losses[-1], opt.norm[0].item(), nuq.nuq_last_error_flags()))
