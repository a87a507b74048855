"""The loss is a tensor of its own, as cross_entropy's is: a program may scale or mask it in place, before or after it is detached.

The module is Python around two entry points; here plain torch stands in for those, on the CPU.  On the device the entry points
themselves are called."""
import pytest
import torch

import paper_1908_06077_amd.loss as loss_module
from paper_1908_06077_amd.loss import linear_cross_entropy

IGNORED = -100


def stand_in_forward(x, w, target, ignore, smoothing, loss, lse, mean, workspace):
    assert loss.is_contiguous() and loss.numel() == lse.numel() == target.numel()
    z = x.reshape(-1, x.shape[-1]) @ w.t()
    t = target.reshape(-1)
    lse.copy_(torch.logsumexp(z, 1))
    each = lse - (1 - smoothing) * z.gather(1, t.clamp(min=0)[:, None])[:, 0] - smoothing * z.mean(1)
    loss.copy_(torch.where(t == ignore, 0.0, each).view(loss.shape))
    if mean is not None:
        count = int((t != ignore).sum())
        mean[1] = 1.0 / count
        mean[0] = loss.sum() * mean[1]


def stand_in_backward(x, w, target, ignore, smoothing, lse, grad, mean, dx, dw, workspace):
    rows = x.reshape(-1, x.shape[-1])
    t = target.reshape(-1)
    d = (rows @ w.t() - lse.reshape(-1, 1)).exp() - smoothing / w.shape[0]
    d[torch.arange(len(t)), t.clamp(min=0)] -= 1 - smoothing
    d = d * torch.where(t == ignore, 0.0, grad.reshape(-1) * (1.0 if mean is None else mean[1]))[:, None]
    if dx is not None:
        dx.copy_((d @ w).view(dx.shape))
    if dw is not None:
        dw.copy_(d.t() @ rows)


@pytest.fixture(params=["cpu", pytest.param("cuda:0", marks=pytest.mark.gpu)])
def device(request, monkeypatch):
    if request.param == "cpu":
        monkeypatch.setattr(loss_module.nuq, "nuq_linear_cross_entropy_forward", stand_in_forward)
        monkeypatch.setattr(loss_module.nuq, "nuq_linear_cross_entropy_backward", stand_in_backward)
        monkeypatch.setattr(loss_module, "_workspace", lambda *a: None)
    return request.param


def leaves(device):
    gen = torch.Generator().manual_seed(1)
    x, w = torch.randn(3, 5, 24, generator=gen), torch.randn(70, 24, generator=gen)
    target = torch.randint(0, 70, (3, 5), generator=gen)
    target[1, 2] = IGNORED
    return x.to(device).requires_grad_(), w.to(device).requires_grad_(), target.to(device)


def gradients(device, reduction, change):
    x, w, target = leaves(device)
    loss = linear_cross_entropy(x, w, target, smoothing=0.1, reduction=reduction)
    loss = change(loss)
    loss.sum().backward()
    return loss.detach().clone(), x.grad, w.grad


@pytest.mark.parametrize("reduction", ["mean", "none"])
def test_scaled_in_place(device, reduction):
    """By a power of two, so that the gradients are the same bits as out of place."""
    def in_place(loss):
        loss /= 4
        return loss
    for a, b in zip(gradients(device, reduction, in_place), gradients(device, reduction, lambda loss: loss / 4)):
        assert torch.equal(a, b)


def test_masked_in_place(device):
    mask = (torch.arange(15, device=device) % 3 != 0).float().view(3, 5)

    def in_place(loss):
        loss *= mask
        return loss
    for a, b in zip(gradients(device, "none", in_place), gradients(device, "none", lambda loss: loss * mask)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("reduction", ["mean", "none"])
def test_changed_after_it_was_detached(device, reduction):
    """What a program does to the value, say for its log, does not reach the gradients."""
    def after(loss):
        out = loss * 1.0
        loss.detach().mul_(1e6)
        return out
    for a, b in zip(gradients(device, reduction, after), gradients(device, reduction, lambda loss: loss * 1.0)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("reduction", ["mean", "none"])
def test_no_view(device, reduction):
    x, w, target = leaves(device)
    loss = linear_cross_entropy(x, w, target, reduction=reduction)
    assert not loss._is_view() and loss.shape == (() if reduction == "mean" else target.shape)
    with torch.no_grad():
        loss = linear_cross_entropy(x, w, target, reduction=reduction)
        loss.zero_()
