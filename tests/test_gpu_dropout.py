"""Dropout: the mask from its definition, results rounded once, and what autograd and graphs make of it.

Bars.  Where nothing is added the result is one product in fp32 (the factor itself rounded to fp32: 2^-24), rounded to the type;
with a residual one more rounding of the sum: three roundings in fp32 of what is added and half a unit of the type."""
import numpy as np
import pytest
import torch

from drop_util import factors, kept

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")
U = 2.0 ** -24
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
HALF_UNIT = {F32: 2.0 ** -24, BF16: 2.0 ** -8, F16: 2.0 ** -11}
LEAST = {F32: 2.0 ** -148, BF16: 2.0 ** -133, F16: 2.0 ** -24}
SHAPES = [(1, 1), (7, 1), (1, 8), (1, 7), (5, 9), (300, 3), (33, 64), (3, 1001), (128, 1600), (1, 70001), (65, 4099), (2100, 513)]


@pytest.fixture(scope="module")
def nuq():
    import paper_1908_06077_amd
    return paper_1908_06077_amd


def rows_of(rows, hidden, kind, gen, pad=0):
    return torch.randn(rows, hidden + pad, generator=gen, device=DEV).to(kind)[:, pad // 2:pad // 2 + hidden]


def test_the_definition_has_no_bias():
    """A million draws per probability: the share of what is kept is within five standard deviations, also over each column."""
    for p in (0.1, 0.5, 0.9):
        k = kept(4096, 256, p, 1234)
        assert abs(k.mean() - (1 - p)) < 5 * (p * (1 - p) / k.size) ** 0.5
        assert np.abs(k.mean(0) - (1 - p)).max() < 5 * (p * (1 - p) / 4096) ** 0.5
        other = kept(4096, 256, p, 1235)
        assert abs((k & other).mean() - (1 - p) ** 2) < 5 * ((1 - p) ** 2 / k.size) ** 0.5       # seeds are independent


@pytest.mark.parametrize("kind", [F32, BF16, F16])
@pytest.mark.parametrize("rows,hidden", SHAPES)
def test_values(nuq, rows, hidden, kind):
    gen = torch.Generator(device=DEV).manual_seed(rows + hidden)
    for p, pad, stream, seed, step in ((0.25, 0, False, 3, None), (0.1, 3, True, -5, 12), (0.0, 1, True, 1, None), (1.0, 0, True, 2, None),
                                       (0.5, 2, False, 2 ** 64 - 1, -1)):
        x = rows_of(rows, hidden, kind, gen, pad)
        r = rows_of(rows, hidden, kind, gen, pad) if stream else None
        y = torch.full((rows, hidden + pad), 7.0, dtype=kind, device=DEV)
        at = None if step is None else torch.tensor([step], device=DEV)
        nuq.nuq_dropout(x, r, p, seed, at, y[:, :hidden])
        f = factors(rows, hidden, p, seed, step or 0)
        b = x.double() * f
        want = b if r is None else b + r.double()
        bar = 2 * U * b.abs() + (U if stream else 0) * want.abs() + HALF_UNIT[kind] * (1 + 4 * U) * want.abs() + LEAST[kind]
        bar += HALF_UNIT[kind] * 2 * U * b.abs()
        assert float(((y[:, :hidden].double() - want).abs() / bar).max()) <= 1.0
        assert (y[:, hidden:] == 7.0).all()
        if not stream:
            assert torch.equal(y[:, :hidden] == 0, (f == 0) | (x == 0))


def test_what_is_dropped_is_zero_whatever_it_was(nuq):
    rows, hidden = 9, 1001
    x = torch.full((rows, hidden), float("nan"), device=DEV)
    x[1::3], x[2::3] = float("inf"), -float("inf")
    y = torch.empty_like(x)
    nuq.nuq_dropout(x, None, 0.5, 11, None, y)
    k = torch.from_numpy(kept(rows, hidden, 0.5, 11)).to(DEV)
    assert torch.equal(y.isfinite(), ~k) and not y[~k].any()


def test_in_place_and_views_and_no_rows(nuq):
    gen = torch.Generator(device=DEV).manual_seed(1)
    for kind in (F32, BF16):
        x, r = rows_of(37, 1003, kind, gen, 5), rows_of(37, 1003, kind, gen, 5)
        want = torch.empty(37, 1003, dtype=kind, device=DEV)
        nuq.nuq_dropout(x, r, 0.3, 4, None, want)
        for which in (0, 1):
            base = (x, r)[which]._base.clone()
            over = base.as_strided((37, 1003), (1008, 1), 2)
            nuq.nuq_dropout(over if which == 0 else x, over if which else r, 0.3, 4, None, over)
            assert torch.equal(over, want)
    nuq.nuq_dropout(torch.empty(0, 5, device=DEV), None, 0.3, 4, None, torch.empty(0, 5, device=DEV))
    x = torch.randn(2, 3, 40, generator=gen, device=DEV)         # leading dimensions are rows
    y, z = torch.empty_like(x), torch.empty(6, 40, device=DEV)
    nuq.nuq_dropout(x, None, 0.3, 4, None, y)
    nuq.nuq_dropout(x.view(6, 40), None, 0.3, 4, None, z)
    assert torch.equal(y.view(6, 40), z)


def test_offsets_beyond_32_bits(nuq):
    hidden, stride, rows = 1001, (1 << 31) + 17, 3
    flat = torch.zeros(stride * (rows - 1) + hidden, dtype=BF16, device=DEV)
    dense = rows_of(rows, hidden, BF16, torch.Generator(device=DEV).manual_seed(1))
    far = flat.as_strided((rows, hidden), (stride, 1))
    far.copy_(dense)
    y, again = torch.empty_like(dense), torch.empty_like(dense)
    nuq.nuq_dropout(dense, None, 0.2, 9, None, y)
    nuq.nuq_dropout(far, None, 0.2, 9, None, again)
    assert torch.equal(y, again)
    nuq.nuq_dropout(far, None, 0.2, 9, None, far)
    assert torch.equal(far, y)


def test_module(nuq):
    from paper_1908_06077_amd.dropout import Dropout
    drop = Dropout(0.25, seed=5)
    x = torch.randn(4, 6, 50, device=DEV, requires_grad=True)
    r = torch.randn(4, 6, 50, device=DEV, requires_grad=True)
    a, b = drop(x), drop(x)
    assert not torch.equal(a, b)                             # every call draws anew
    y = drop(x, r)
    g = torch.randn_like(y)
    y.backward(g)
    mask = ((y - r).detach().abs() > 1e-6).float() / 0.75
    assert torch.equal(r.grad, g) and float((x.grad - g * mask).abs().max()) <= 4 * U * float(g.abs().max()) / 0.75
    again = Dropout(0.25, seed=5)
    assert torch.equal(again(x), a) and torch.equal(again(x), b)
    drop.eval()
    assert drop(x) is x and torch.equal(drop(x, r), x + r)
    for bad in (lambda: Dropout(1.5), lambda: drop(x, r[0]), lambda: drop(torch.tensor(1.0, device=DEV))):
        with pytest.raises(ValueError):
            bad()


def test_graph_draws_anew_where_its_step_moves(nuq):
    from paper_1908_06077_amd.dropout import Dropout
    step = torch.zeros(1, dtype=torch.int64, device=DEV)
    drop = Dropout(0.5, seed=3, step=step)
    x, eager = torch.randn(64, 1600, device=DEV), []
    first = drop.draws.calls
    y, dx = torch.empty_like(x), torch.empty_like(x)

    def both(seed):
        nuq.nuq_dropout(x, None, 0.5, seed, step, y)
        nuq.nuq_dropout(x, None, 0.5, seed, step, dx)
    seed = drop.draws.next()
    assert drop.draws.calls == first + 1
    both(seed)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(seed)
    for k in range(4):
        step.fill_(k)
        both(seed)
        eager.append(y.clone())
        y.zero_(), dx.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, eager[k]) and torch.equal(dx, y)
    assert len({int((e != 0).sum()) for e in eager}) > 1


def test_module_without_a_seed_draws_from_torch(nuq):
    """Two modules have masks of their own, torch.manual_seed repeats them, and a function that is run again for its gradients has the masks
    of its first run: with and without that the gradients are the same bits."""
    from torch.utils.checkpoint import checkpoint

    from paper_1908_06077_amd.dropout import Dropout
    x = torch.ones(64, 512, device=DEV)
    one, two = Dropout(0.5), Dropout(0.5)
    torch.manual_seed(11)
    a, b = one(x), two(x)
    torch.manual_seed(11)
    assert torch.equal(a, two(x)) and torch.equal(b, one(x))
    agree = (a == b).float().mean().item()                   # of 32768 fair coins: 0.5, six deviations are 0.017
    assert abs(agree - 0.5) < 0.017

    w = torch.randn(512, 512, device=DEV, generator=torch.Generator(DEV).manual_seed(1), requires_grad=True)

    def both(x):
        return two(torch.tanh(one(x) @ w), x)

    grads = []
    for again in (False, True):
        torch.manual_seed(12)
        y = checkpoint(both, x, use_reentrant=False) if again else both(x)
        grads.append(torch.autograd.grad((y * torch.arange(512, device=DEV)).sum(), w)[0])
    assert torch.equal(*grads)
