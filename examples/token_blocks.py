"""A stack of residual blocks over tokens, trained by K simulated workers with coded gradients: dropout behind the embedding, seams with a
norm on either side of the residual sum, gate and dropout, and the loss over the vocabulary without its logits.

    python examples/token_blocks.py [--steps 100] [--dtype bfloat16]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_1908_06077_amd as nuq  # noqa: E402
from paper_1908_06077_amd.dropout import Dropout  # noqa: E402
from paper_1908_06077_amd.loss import LinearCrossEntropy  # noqa: E402
from paper_1908_06077_amd.norm import ResidualNorm  # noqa: E402
from paper_1908_06077_amd.optim import NUQAdamW  # noqa: E402


class TokenBlocks(torch.nn.Module):
    """stream <- stream + gate drop(norm(MLP(norm(stream)))), `depth` times, behind an embedding; the loss of the next token.  dtype: of the
    rows and products; the parameters are fp32."""

    def __init__(self, vocab: int, width: int, depth: int, dropout: float = 0.1, dtype: torch.dtype = torch.float32, seed: int = 0):
        super().__init__()
        self.dtype = dtype
        self.embed = torch.nn.Embedding(vocab, width)
        self.drop = Dropout(dropout, seed=seed)
        self.first = ResidualNorm(width, outer="rms", bias=False)
        self.seams = torch.nn.ModuleList(ResidualNorm(width, inner="rms", outer="rms", bias=False, gate=0.5, dropout=dropout,
                                                      seed=seed + 1 + k) for k in range(depth))
        self.up = torch.nn.ModuleList(torch.nn.Linear(width, 4 * width) for _ in range(depth))
        self.down = torch.nn.ModuleList(torch.nn.Linear(4 * width, width) for _ in range(depth))
        self.head = LinearCrossEntropy(width, vocab)

    def _linear(self, layer, x):
        return torch.nn.functional.linear(x, layer.weight.to(x.dtype), layer.bias.to(x.dtype))

    def forward(self, tokens, target):
        y, stream = self.first(self.drop(self.embed(tokens).to(self.dtype)))
        for up, down, seam in zip(self.up, self.down, self.seams):
            y, stream = seam(self._linear(down, torch.nn.functional.gelu(self._linear(up, y))), stream)
        return self.head(y, target)


def groups(model, decay=0.1):
    """Weight decay for matrices alone."""
    params = list(model.parameters())
    return [{"params": [p for p in params if p.dim() > 1], "weight_decay": decay},
            {"params": [p for p in params if p.dim() <= 1], "weight_decay": 0.0}]


def train(steps=100, K=4, vocab=500, width=96, depth=2, batch=8, length=32, dtype=torch.float32, lr=2e-3, seed=3):
    """(losses, optimizer) of `steps` steps on sequences in which a token follows from the one before it; the first is padding now and
    then, whose loss does not count."""
    dev = torch.device("cuda")
    torch.manual_seed(seed)
    model = TokenBlocks(vocab, width, depth, dtype=dtype, seed=seed).to(dev)
    opt = NUQAdamW(groups(model), K=K, lr=lr, betas=(0.9, 0.95), bucket=512, s=4, max_norm=1.0, seed=seed)
    g = torch.Generator(device=dev).manual_seed(seed)
    follows = torch.randperm(vocab, generator=g, device=dev)
    losses = []
    for _ in range(steps):
        step = []
        for k in range(K):
            tokens = torch.randint(0, vocab, (batch, length), generator=g, device=dev)
            target = follows[tokens]
            target[:, 0] = torch.where(tokens[:, 0] % 3 == 0, -100, target[:, 0])
            with opt.worker(k):
                loss = model(tokens, target)
                loss.backward()
            step.append(loss.detach())
        opt.step()
        losses.append(torch.stack(step).mean())
    return torch.stack(losses).tolist(), opt


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=100)
    ap.add_argument("--dtype", default="float32", choices=("float32", "bfloat16", "float16"))
    a = ap.parse_args()
    losses, opt = train(a.steps, dtype=getattr(torch, a.dtype))
    for t in range(0, len(losses), max(1, len(losses) // 10)):
        print("step %4d  loss %.4f" % (t, losses[t]))
    print("last       loss %.4f, norm of the last average %.4f, flags %d" % (losses[-1], opt.norm[0].item(), nuq.nuq_last_error_flags()))
