"""ResidualNorm where only the stream is used further: the norm's own gradient is 0, also of rows that it has no finite value for."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("inner,outer", [(None, "layer"), (None, "rms"), ("rms", "layer"), ("layer", "rms")])
@pytest.mark.parametrize("hidden", [5, 72, 1003, 9001])
def test_norm_that_is_not_used(hidden, inner, outer, kind):
    """Without the outer norm the gradients of the same call are what they should be; stream rows of equal elements (variance 0, eps 0), of
    infinities and of NaN do not reach them."""
    from paper_1908_06077_amd.norm import ResidualNorm
    rows = 7
    gen = torch.Generator(device=DEV).manual_seed(hidden)
    x, r, g = (torch.randn(rows, hidden, generator=gen, device=DEV).to(kind) for _ in range(3))
    r[1], x[1] = 0.0, 0.0
    r[2, 0], r[3, hidden - 1], r[4, 1] = float("inf"), -float("inf"), float("nan")
    both = []
    for norm in (outer, None):
        if norm is None and inner is None:
            break                                            # (a norm there has to be: the formula below)
        m = ResidualNorm(hidden, inner=inner, outer=norm, gate=0.5, scale=0.7, residual_scale=0.5, dropout=0.3, seed=3,
                         eps=0.0 if inner is None else 1e-3, device=DEV)
        if norm:
            m.outer_weight.data[0] = float("inf")
        a, b = x.clone().requires_grad_(), r.clone().requires_grad_()
        out = m(a, b)
        (out[1] if norm else out).backward(g.t().contiguous().t())           # (of rows that do not stand as the kernels take them)
        assert not norm or (not m.outer_weight.grad.any() and not m.outer_bias.grad.any())
        both.append([a.grad, b.grad, m.gate.grad] + ([m.inner_weight.grad, m.inner_bias.grad] if inner else []))
    assert all(t.isfinite().all() for t in both[0])
    assert torch.equal(both[0][1], (g.float() * 0.5).to(kind))
    if inner is not None:
        assert all(torch.equal(p, q) for p, q in zip(*both))
    else:
        from drop_util import factors
        seed = type(m.draws)(0.3, 3, None).next()
        want = g.double() * 0.5 * 0.7 * factors(rows, hidden, 0.3, seed)      # two roundings of the factors, one of the product
        half = torch.finfo(kind).eps / 2
        assert bool(((both[0][0].double() - want).abs() <= (half + 4 * 2.0 ** -24) * 1.01 * want.abs() + 2.0 ** -24 * (kind == torch.float16)).all())
