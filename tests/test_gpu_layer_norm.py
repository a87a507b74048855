"""Layer norm forward and backward against their formulas in 64 bits, and the module against autograd's rules.

Bars.  u = 2^-24.  A sum over a row passes through at most 64 additions in any order that the kernels use (32 elements per
thread, six steps over a wave, sixteen waves): 64 u of the mean magnitude.  The mean's error moves n by that times rstd; the
variance is a mean of centred squares, so n's relative error is half of 64 u and a few roundings.  Results are rounded to their
type: half a unit of its last place.  Weight gradients add rows / 512 elements per workgroup and 512 of those: 64 + rows / 512
roundings of the summed magnitudes."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")
U = 2.0 ** -24
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
HALF_UNIT = {F32: 2.0 ** -24, BF16: 2.0 ** -8 * 1.01, F16: 2.0 ** -11 * 1.01}
LEAST = {F32: 2.0 ** -140, BF16: 2.0 ** -126, F16: 2.0 ** -24}
SHAPES = [(1, 1), (5, 1), (3, 2), (70, 7), (1, 8), (33, 9), (300, 31), (17, 32), (5, 33), (130, 64), (9, 127), (4, 128), (2, 129),
          (65, 255), (3, 257), (7, 511), (2100, 512), (5, 513), (1, 1000), (6, 1024), (3, 1025), (1, 1600), (601, 1600), (4, 2047),
          (2, 2049), (3, 4096), (5, 4099), (2, 8192), (3, 8195), (2, 12288), (1, 16384), (2, 16389), (3, 20001)]
KINDS = [(F32, F32), (BF16, F32), (BF16, BF16), (F16, F32), (F16, F16)]


@pytest.fixture(scope="module")
def nuq():
    import paper_1908_06077_amd
    return paper_1908_06077_amd


def rows_of(rows, hidden, kind, gen, pad=0, scale=1.0, shift=0.0):
    x = torch.randn(rows, hidden + pad, generator=gen, device=DEV) * scale + shift * torch.randn(rows, 1, generator=gen, device=DEV)
    return x.to(kind)[:, pad // 2:pad // 2 + hidden]


def close(got, want, bar):
    got = got.double()
    worst = float(((got - want).abs() / bar).max()) if got.numel() else 0.0
    assert worst <= 1.0, worst


def forward_formula(s, weight, bias, eps, kind):
    """(y, mean, rstd, bars) in fp64."""
    s = s.double()
    mean = s.mean(1, keepdim=True)
    var = (s - mean).square().mean(1, keepdim=True)
    rstd = (var + eps).rsqrt()
    top = s.abs().mean(1, keepdim=True)
    w = torch.ones(s.shape[1], dtype=torch.float64, device=DEV) if weight is None else weight.double()
    b = torch.zeros(s.shape[1], dtype=torch.float64, device=DEV) if bias is None else bias.double()
    n = (s - mean) * rstd
    bar_mean = 65 * U * top + 2.0 ** -148
    bar_rstd = rstd * (36 * U + 4 * (bar_mean * rstd) ** 2)
    bar_n = bar_mean * rstd + 40 * U * n.abs() + 4 * n.abs() * (bar_mean * rstd) ** 2
    y = n * w + b
    bar_y = bar_n * w.abs() + 2 * U * (n * w).abs() + HALF_UNIT[kind] * (y.abs() + bar_n * w.abs()) + U * y.abs() + LEAST[kind]
    return y, mean[:, 0], rstd[:, 0], bar_y, bar_mean[:, 0], bar_rstd[:, 0]


@pytest.mark.parametrize("kind,weights", KINDS)
@pytest.mark.parametrize("rows,hidden", SHAPES)
def test_forward(nuq, rows, hidden, kind, weights):
    gen = torch.Generator(device=DEV).manual_seed(rows * 31 + hidden)
    vector = lambda at: (at + 0.3 * torch.randn(hidden + 1, generator=gen, device=DEV)).to(weights)[1:].contiguous()  # noqa: E731
    eps = 1e-5
    for pad, affine, stream in ((0, 2, False), (0, 2, True), (3, 1, True), (5, 0, False)):
        x = rows_of(rows, hidden, kind, gen, pad, 2.0, 3.0)
        weight, bias = vector(1.0) if affine else None, vector(0.0) if affine == 2 else None
        residual = rows_of(rows, hidden, kind, gen, pad) if stream else None
        y = torch.full((rows, hidden + pad), 7.0, dtype=kind, device=DEV)
        total = torch.full((rows, hidden + pad), 7.0, dtype=kind, device=DEV) if stream else None
        mean, rstd = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
        nuq.nuq_layer_norm_forward(x, residual, weight, bias, eps, total[:, :hidden] if stream else None, y[:, :hidden], mean, rstd)
        s = x
        if stream:
            s = (x.float() + residual.float()).to(kind)
            assert torch.equal(total[:, :hidden], s) and (total[:, hidden:] == 7.0).all()
        want = forward_formula(s, weight, bias, eps, kind)
        close(y[:, :hidden], want[0], want[3])
        close(mean, want[1], want[4])
        close(rstd, want[2], want[5])
        assert (y[:, hidden:] == 7.0).all()
        plain = torch.empty(rows, hidden, dtype=kind, device=DEV)
        nuq.nuq_layer_norm_forward(s, None, weight, bias, eps, None, plain, None, None)      # without statistics: the same
        assert torch.equal(plain, y[:, :hidden])


@pytest.mark.parametrize("kind,weights", KINDS)
@pytest.mark.parametrize("rows,hidden", SHAPES)
def test_backward(nuq, rows, hidden, kind, weights):
    gen = torch.Generator(device=DEV).manual_seed(rows * 17 + hidden)
    for pad, affine, stream in ((0, 2, False), (3, 2, True), (5, 1, False), (0, 0, True)):
        x, dy = rows_of(rows, hidden, kind, gen, pad, 2.0, 3.0), rows_of(rows, hidden, kind, gen, pad, 0.5)
        weight = (1.0 + 0.3 * torch.randn(hidden, generator=gen, device=DEV)).to(weights) if affine else None
        add = rows_of(rows, hidden, kind, gen, pad) if stream else None
        s = x.double()
        mean = s.mean(1).float()
        rstd = (s.var(1, correction=0) + 1e-5).rsqrt().float()
        dx = torch.full((rows, hidden + pad), 7.0, dtype=kind, device=DEV)
        dw = torch.empty(hidden, dtype=weights, device=DEV) if affine else None
        db = torch.empty(hidden, dtype=weights, device=DEV) if affine == 2 else None
        ws = torch.empty(nuq.nuq_layer_norm_workspace_bytes(rows, hidden), dtype=torch.uint8, device=DEV) if affine else None
        nuq.nuq_layer_norm_backward(dy, x, weight, mean, rstd, add, dx[:, :hidden], dw, db, ws)
        m, r = mean.double()[:, None], rstd.double()[:, None]
        n, d = (s - m) * r, dy.double()
        many = (64 + rows / 512) * U
        if affine:
            close(dw, (d * n).sum(0), (d * n).abs().sum(0) * (many + 4 * U) + (d * n).sum(0).abs() * HALF_UNIT[weights] + LEAST[weights])
        if affine == 2:
            close(db, d.sum(0), d.abs().sum(0) * many + d.sum(0).abs() * HALF_UNIT[weights] + LEAST[weights])
        d = d * weight.double() if affine else d
        s1, s2 = d.mean(1, keepdim=True), (d * n).mean(1, keepdim=True)
        a1, a2 = d.abs().mean(1, keepdim=True), (d * n).abs().mean(1, keepdim=True)
        want = r * (d - s1 - n * s2)
        bar = r * (68 * U * (a1 + n.abs() * a2) + 8 * U * (d.abs() + s1.abs() + (n * s2).abs()))
        if stream:
            want = want + add.double()
            bar = bar + U * want.abs()
        close(dx[:, :hidden], want, bar + HALF_UNIT[kind] * (want.abs() + bar) + LEAST[kind])
        assert (dx[:, hidden:] == 7.0).all()
        if affine:                                           # without the sums: the same rows
            again = torch.empty(rows, hidden, dtype=kind, device=DEV)
            nuq.nuq_layer_norm_backward(dy, x, weight, mean, rstd, add, again, None, None, None)
            assert torch.equal(again, dx[:, :hidden])


@pytest.mark.parametrize("rows,hidden", [(20_001, 40), (70_000, 9), (4097, 640), (9000, 2050)])
def test_weight_gradients_of_many_rows(nuq, rows, hidden):
    gen = torch.Generator(device=DEV).manual_seed(rows)
    x, dy = rows_of(rows, hidden, F32, gen), rows_of(rows, hidden, F32, gen)
    mean, rstd = torch.zeros(rows, device=DEV), torch.ones(rows, device=DEV)
    ws = torch.empty(nuq.nuq_layer_norm_workspace_bytes(rows, hidden), dtype=torch.uint8, device=DEV)
    dx, first = torch.empty_like(x), None
    for _ in range(2):
        dw, db = torch.empty(hidden, device=DEV), torch.empty(hidden, device=DEV)
        nuq.nuq_layer_norm_backward(dy, x, None, mean, rstd, None, dx, dw, db, ws)
        p = x.double() * dy.double()
        many = (68 + rows / 512) * U
        close(dw, p.sum(0), p.abs().sum(0) * many)
        close(db, dy.double().sum(0), dy.double().abs().sum(0) * many)
        first = first or (dw, db)
        assert torch.equal(first[0], dw) and torch.equal(first[1], db)       # a fixed order: the same bits


def test_rows_far_from_zero_and_of_one_value(nuq):
    """A mean a thousand times the spread leaves the variance exact to the mean's own rounding; a constant row gives the bias."""
    hidden = 1600
    gen = torch.Generator(device=DEV).manual_seed(3)
    x = 1000.0 + torch.randn(4, hidden, generator=gen, device=DEV)
    x[1] = 0.1
    x[2] = 0.0
    bias = torch.randn(hidden, generator=gen, device=DEV)
    y, mean, rstd = torch.empty_like(x), torch.empty(4, device=DEV), torch.empty(4, device=DEV)
    nuq.nuq_layer_norm_forward(x, None, None, bias, 1e-5, None, y, mean, rstd)
    want = forward_formula(x, None, bias, 1e-5, F32)
    close(y, want[0], want[3])
    close(rstd, want[2], want[5])
    assert torch.equal(y[2], bias)


def test_infinite_and_missing_values_stay_in_their_rows(nuq):
    hidden = 700
    gen = torch.Generator(device=DEV).manual_seed(4)
    x = torch.randn(40, hidden, generator=gen, device=DEV)
    clean = torch.empty_like(x)
    nuq.nuq_layer_norm_forward(x, None, None, None, 1e-5, None, clean, None, None)
    x[5, 3], x[9, 699], x[20, 0] = float("nan"), float("inf"), -float("inf")
    y = torch.empty_like(x)
    nuq.nuq_layer_norm_forward(x, None, None, None, 1e-5, None, y, None, None)
    bad = [5, 9, 20]
    fine = [r for r in range(40) if r not in bad]
    assert torch.equal(y[fine], clean[fine]) and not torch.isfinite(y[bad]).any()


def test_no_rows(nuq):
    x = torch.empty(0, 33, device=DEV)
    stats = torch.empty(0, device=DEV)
    nuq.nuq_layer_norm_forward(x, None, None, None, 1e-5, None, torch.empty_like(x), stats, stats)
    dw, db = torch.full((33,), 7.0, device=DEV), torch.full((33,), 7.0, device=DEV)
    nuq.nuq_layer_norm_backward(x, x, None, stats, stats, None, torch.empty_like(x), dw, db, torch.empty(8, dtype=torch.uint8, device=DEV))
    assert not dw.any() and not db.any()                     # sums over no rows


def test_results_may_stand_where_the_rows_stood(nuq):
    for hidden in (100, 1600, 20001):
        gen = torch.Generator(device=DEV).manual_seed(hidden)
        x, dy = rows_of(9, hidden, BF16, gen), rows_of(9, hidden, BF16, gen)
        y, mean, rstd = torch.empty_like(x), torch.empty(9, device=DEV), torch.empty(9, device=DEV)
        nuq.nuq_layer_norm_forward(x, None, None, None, 1e-5, None, y, mean, rstd)
        ws = torch.empty(nuq.nuq_layer_norm_workspace_bytes(9, hidden), dtype=torch.uint8, device=DEV)
        out = [[torch.empty_like(x), torch.empty(hidden, device=DEV), torch.empty(hidden, device=DEV)] for _ in range(2)]
        nuq.nuq_layer_norm_backward(dy, x, None, mean, rstd, None, *out[0], ws)
        out[1][0] = dy
        nuq.nuq_layer_norm_backward(dy, x, None, mean, rstd, None, *out[1], ws)
        assert all(torch.equal(a, b) for a, b in zip(*out))
        nuq.nuq_layer_norm_forward(x, None, None, None, 1e-5, None, x, None, None)
        assert torch.equal(x, y)
        for at in (0, 1):                                    # the sum in the place of either
            r = rows_of(9, hidden, BF16, gen)
            s = (y.float() + r.float()).bfloat16()
            both = [y.clone(), r]
            out = torch.empty_like(y)
            nuq.nuq_layer_norm_forward(both[0], both[1], None, None, 1e-5, both[at], out, None, None)
            want = torch.empty_like(y)
            nuq.nuq_layer_norm_forward(s, None, None, None, 1e-5, None, want, None, None)
            assert torch.equal(both[at], s) and torch.equal(out, want)


def test_offsets_beyond_32_bits(nuq):
    """Rows at a stride that puts the last of them beyond 2^32 elements."""
    hidden, stride, rows = 1001, (1 << 31) + 17, 3
    flat = torch.zeros(stride * (rows - 1) + hidden, dtype=BF16, device=DEV)
    gen = torch.Generator(device=DEV).manual_seed(1)
    dense = rows_of(rows, hidden, BF16, gen)
    far = flat.as_strided((rows, hidden), (stride, 1))
    far.copy_(dense)
    y, again = torch.empty_like(dense), torch.empty_like(dense)
    mean, rstd = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    nuq.nuq_layer_norm_forward(dense, None, None, None, 1e-5, None, y, mean, rstd)
    nuq.nuq_layer_norm_forward(far, None, None, None, 1e-5, None, again, None, None)
    assert torch.equal(y, again)
    nuq.nuq_layer_norm_forward(far, None, None, None, 1e-5, None, far, None, None)
    assert torch.equal(far, y)


# ---------------------------------------------------------------------------------------- the module

def module(hidden, weights=F32, **kw):
    from paper_1908_06077_amd.norm import LayerNorm
    m = LayerNorm(hidden, device=DEV, dtype=weights, **kw)
    gen = torch.Generator(device=DEV).manual_seed(hidden)
    for p in m.parameters():
        p.data.add_((0.2 * torch.randn(hidden, generator=gen, device=DEV)).to(weights))
    return m


def test_module_gradients_against_differences(nuq):
    """Central differences of the formula in 64 bits, on a few elements of every input."""
    hidden, rows, h = 37, 6, 1e-5
    m = module(hidden)
    gen = torch.Generator(device=DEV).manual_seed(2)
    x, r, gy, gt = (torch.randn(rows, hidden, generator=gen, device=DEV) for _ in range(4))
    x.requires_grad_()
    r.requires_grad_()
    y, total = m(x, r)
    ((y * gy).sum() + (total * gt).sum()).backward()

    def loss(x, r, w, b):
        s = x + r
        n = (s - s.mean(1, keepdim=True)) * (s.var(1, correction=0, keepdim=True) + m.eps).rsqrt()
        return float(((n * w + b) * gy.double()).sum() + (s * gt.double()).sum())
    inputs = [t.detach().double() for t in (x, r, m.weight, m.bias)]
    for k, grad in enumerate((x.grad, r.grad, m.weight.grad, m.bias.grad)):
        for at in range(0, grad.numel(), 7):
            ends = []
            for sign in (1, -1):
                moved = [t.clone() for t in inputs]
                moved[k].view(-1)[at] += sign * h
                ends.append(loss(*moved))
            slope = (ends[0] - ends[1]) / (2 * h)            # error: h^2 times a third derivative of order ten, rounding 1e-13 / h
            assert abs(float(grad.view(-1)[at]) - slope) <= 1e-5 * (1.0 + abs(slope)), (k, at)


def test_module_accepts_what_autograd_hands_it(nuq):
    m = module(24)
    gen = torch.Generator(device=DEV).manual_seed(5)
    base = torch.randn(24, 4, 3, generator=gen, device=DEV)
    x = base.permute(2, 1, 0).requires_grad_()               # rows that are not contiguous
    y = m(x)
    y.sum().backward()                                       # a gradient of stride zero
    ref = torch.nn.LayerNorm(24).double()
    ref.load_state_dict({k: v.cpu().double() for k, v in m.state_dict().items()})
    xr = x.detach().cpu().double().requires_grad_()
    ref(xr).sum().backward()
    bar = 1e-5
    assert torch.allclose(y.detach().cpu().double(), ref(xr).detach(), rtol=0, atol=bar)
    assert torch.allclose(m.weight.grad.cpu().double(), ref.weight.grad, rtol=0, atol=bar)
    assert torch.allclose(m.bias.grad.cpu().double(), ref.bias.grad, rtol=0, atol=bar)
    # the sum alone is used, or the norm alone; nothing that needs no gradient gets one
    a, b = (torch.randn(3, 24, generator=gen, device=DEV, requires_grad=True) for _ in range(2))
    m.zero_grad()
    m(a, b)[1].sum().backward()
    assert (a.grad == 1).all() and (b.grad == 1).all() and m.weight.grad is None
    frozen = module(24).requires_grad_(False)
    out, _ = frozen(a, b.detach())
    out.square().sum().backward()
    assert frozen.weight.grad is None
    for kw in (dict(bias=False), dict(elementwise_affine=False)):
        k = module(24, **kw)
        assert k.bias is None
        k(a).sum().backward()
    with pytest.raises(ValueError):
        m(torch.zeros(2, 25, device=DEV))
    with pytest.raises(ValueError):
        m(torch.zeros(2, 24, device=DEV), torch.zeros(1, 24, device=DEV))


def test_module_in_sixteen_bits(nuq):
    for kind, weights in ((BF16, F32), (BF16, BF16), (F16, F16)):
        m = module(200, weights)
        x = torch.randn(5, 7, 200, device=DEV, generator=torch.Generator(device=DEV).manual_seed(1)).to(kind).requires_grad_()
        y = m(x)
        assert y.dtype == kind and y.shape == x.shape
        y.float().square().sum().backward()
        assert x.grad.dtype == kind and m.weight.grad.dtype == weights and torch.isfinite(x.grad).all()


def test_forward_and_backward_replay_in_a_graph(nuq):
    m = module(1600)
    x = torch.randn(300, 1600, device=DEV)
    dy, dx, dw, db, y = (torch.empty_like(x) for _ in range(5))
    dw, db = dw[0].clone(), db[0].clone()
    dy.normal_()
    mean, rstd = torch.empty(300, device=DEV), torch.empty(300, device=DEV)
    ws = torch.empty(nuq.nuq_layer_norm_workspace_bytes(300, 1600), dtype=torch.uint8, device=DEV)

    def both():
        nuq.nuq_layer_norm_forward(x, None, m.weight.detach(), m.bias.detach(), 1e-5, None, y, mean, rstd)
        nuq.nuq_layer_norm_backward(dy, x, m.weight.detach(), mean, rstd, None, dx, dw, db, ws)
    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for _ in range(4):
        x.normal_()
        both()
        want = [t.clone() for t in (y, dx, dw, db)]
        for t in (y, dx, dw, db):
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (y, dx, dw, db)))
