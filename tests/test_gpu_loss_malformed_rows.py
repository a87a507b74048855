"""Rows whose target lies outside the vocabulary: their gradient is 0, whatever gradient comes back for their loss, which is NaN."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")
BAD = [float("nan"), float("inf"), 3e38, -1e30, 0.0]


@pytest.fixture(scope="module")
def nuq():
    import paper_1908_06077_amd
    return paper_1908_06077_amd


def inputs(rows, hidden, vocab, kind, seed=1):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    x, w = (torch.randn(n, hidden, generator=gen, device=DEV).to(kind) for n in (rows, vocab))
    return x, w, torch.randint(0, vocab, (rows,), generator=gen, device=DEV), torch.rand(rows, generator=gen, device=DEV) + 0.5


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows", [3, 70, 1500])
def test_gradient_of_a_row_that_does_not_count(nuq, rows, kind):
    """The same bits as where the row is ignored, which the other tests compare with the formula."""
    x, w, target, grad = inputs(rows, 72, 301, kind)
    out = []
    ws = torch.empty(nuq.nuq_linear_cross_entropy_workspace_bytes(x, w, True), dtype=torch.uint8, device=DEV)
    lse = torch.logsumexp(x.float() @ w.float().t(), 1)
    nuq.nuq_last_error_flags()
    for bad in [-100, 301, -1, 2 ** 40]:
        for value in BAD if bad != -100 else BAD[-1:]:
            t, g = target.clone(), grad.clone()
            t[rows // 2], g[rows // 2] = bad, value
            dx, dw = torch.empty_like(x), torch.empty_like(w)
            nuq.nuq_linear_cross_entropy_backward(x, w, t, -100, 0.0, lse, g, None, dx, dw, ws)
            assert nuq.nuq_last_error_flags() == (0 if bad == -100 else nuq.FLAG_MALFORMED)
            out.append((dx, dw))
            assert not dx[rows // 2].any() and dw.isfinite().all(), (bad, value)
            assert torch.equal(dx, out[0][0]) and torch.equal(dw, out[0][1]), (bad, value)


def test_masked_losses(nuq):
    """A loss that makes a NaN of the malformed row's own gradient, with the row taken out of the sum."""
    from paper_1908_06077_amd.loss import linear_cross_entropy
    x, w, target, _ = inputs(40, 64, 200, torch.float32)
    got = []
    for bad in (-100, 200):
        t = target.clone()
        t[7] = bad
        a, b = x.clone().requires_grad_(), w.clone().requires_grad_()
        losses = linear_cross_entropy(a, b, t, reduction="none").square()     # its slope: 2 loss, NaN in row 7
        keep = torch.arange(40, device=DEV) != 7
        torch.where(keep, losses, torch.zeros_like(losses)).sum().backward()
        got.append((a.grad, b.grad))
    nuq.nuq_last_error_flags()
    assert got[1][1].isfinite().all() and all(torch.equal(p, q) for p, q in zip(*got))
