"""Dropout, the residual norm and the loss together, as a step of the example's model uses them: its loss and every gradient against the
formulas in 64 bits with the masks from their definition, its training step with coded gradients, and two streams at once."""
import os
import sys

import pytest
import torch

from drop_util import factors

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def seeds_of(draws):
    """The seed of a module's next call, which is not used up."""
    return type(draws)(draws.p, draws.seed, None).next() if draws.calls == 0 else None


def rms(s, weight, eps):
    return s * (s.square().mean(-1, keepdim=True) + eps).rsqrt() * weight


def formula(model, tokens, target):
    """The loss of the model's first call in training, in fp64, and the parameters that it is of."""
    p = {k: v.detach().double().requires_grad_() for k, v in model.named_parameters()}
    rows, width = tokens.numel(), model.embed.weight.shape[1]
    drop = lambda draws: factors(rows, width, draws.p, seeds_of(draws))  # noqa: E731
    stream = torch.nn.functional.embedding(tokens.view(-1), p["embed.weight"]) * drop(model.drop.draws)
    y = rms(stream, p["first.outer_weight"], model.first.eps)
    for k, seam in enumerate(model.seams):
        name = lambda x: p["seams.%d.%s" % (k, x)]  # noqa: E731
        h = torch.nn.functional.gelu(y @ p["up.%d.weight" % k].t() + p["up.%d.bias" % k])
        b = rms(h @ p["down.%d.weight" % k].t() + p["down.%d.bias" % k], name("inner_weight"), seam.eps)
        stream = stream + b * name("gate") * drop(seam.draws)
        y = rms(stream, name("outer_weight"), seam.eps)
    return torch.nn.functional.cross_entropy(y @ p["head.weight"].t(), target.view(-1)), p


def test_loss_and_gradients_of_a_step():
    """In fp32.  The products between the operators are the library's: sums of at most 4 x 72 terms, so that some five hundred roundings of
    2^-24 of the magnitudes lie between the formula and a result; gradients are compared with the largest of their tensor."""
    import token_blocks
    torch.manual_seed(1)
    model = token_blocks.TokenBlocks(311, 72, 2, dropout=0.2, seed=5).to(DEV)
    for q in model.parameters():
        if q.dim() == 1:
            q.data.add_(0.1 * torch.randn_like(q))
    tokens, target = torch.randint(0, 311, (5, 13), device=DEV), torch.randint(0, 311, (5, 13), device=DEV)
    target[2, 3:] = -100
    want, p = formula(model, tokens, target)
    want.backward()
    loss = model(tokens, target)
    loss.backward()
    assert abs(float(loss.detach()) - float(want.detach())) <= 512 * 2.0 ** -24 * float(want.detach())
    for name, q in model.named_parameters():
        exact = p[name].grad
        assert float((q.grad.double() - exact).abs().max()) <= 4 * 512 * 2.0 ** -24 * float(exact.abs().max()), name


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_example_runs(dtype):
    import paper_1908_06077_amd as nuq
    import token_blocks
    losses, opt = token_blocks.train(steps=5, vocab=301, width=64, depth=2, batch=3, length=17, dtype=dtype)
    assert len(losses) == 5 and all(x == x and x < 20.0 for x in losses)
    assert bool(torch.isfinite(opt.norm).all()) and nuq.nuq_last_error_flags() == 0


def test_two_streams_at_once():
    """The same step on two streams, with workspaces of their own: each as if it were alone."""
    import token_blocks
    torch.manual_seed(2)
    models = [token_blocks.TokenBlocks(911, 128, 1, dropout=0.1, seed=k).to(DEV) for k in (1, 2)]
    tokens, target = torch.randint(0, 911, (2, 8, 64), device=DEV), torch.randint(0, 911, (2, 8, 64), device=DEV)

    def step(k):
        model = models[k]
        for m in model.modules():
            if hasattr(m, "draws"):
                m.draws.calls = 0
        model.zero_grad()
        loss = model(tokens[k], target[k])
        loss.backward()
        return [loss.detach(), *[q.grad for n, q in model.named_parameters() if not n.startswith("embed")]]     # (torch adds rows in any order)
    want = [step(k) for k in (0, 1)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for k, s in enumerate(streams):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            got.append(step(k))
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        for x, y in zip(a, b):                               # (the products between may take another kernel beside other work)
            assert float((x - y).abs().max()) <= 1e-5 * float(x.abs().max())
