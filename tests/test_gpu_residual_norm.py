"""The norms around a block's residual sum, forward and backward, against their formulas in 64 bits.

Bars.  u = 2^-24.  A sum over a row passes through at most 64 additions (16 elements per thread, six steps over a wave, sixteen
waves): 64 u of the mean magnitude, 66 with the division and the rounding of what is summed.  Every product and sum beside it is one
rounding.  total and y are rounded to their type: half a unit.  y is compared with the formula on the kernel's own total, whose
statistics it is made of.  Backward the forward's statistics are inputs; sums over rows take at most rows / 256 + 64 roundings of the
summed magnitudes.  An error of a factor goes through the products behind it: the bars below follow the formula line by line."""
import pytest
import torch

from drop_util import factors

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")
U = 2.0 ** -24
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
HALF_UNIT = {F32: 2.0 ** -24, BF16: 2.0 ** -8, F16: 2.0 ** -11}
LEAST = {F32: 2.0 ** -140, BF16: 2.0 ** -126, F16: 2.0 ** -24}
KINDS = [(F32, F32), (BF16, F32), (BF16, BF16), (F16, F32), (F16, F16)]
SHAPES = [(1, 1), (5, 2), (3, 3), (70, 7), (1, 8), (33, 9), (300, 31), (5, 33), (130, 64), (9, 127), (4, 129), (65, 255), (7, 511),
          (2100, 512), (5, 513), (1, 1000), (3, 1025), (1, 1600), (601, 1600), (4, 2047), (2, 2049), (3, 4096), (5, 4099), (2, 8192),
          (70, 8195), (2, 12288), (3, 16384)]
NORMS = [("layer", "layer"), ("rms", "rms"), ("none", "layer"), ("none", "rms"), ("rms", "none"), ("layer", "none"), ("layer", "rms")]
EPS = 1e-5


@pytest.fixture(scope="module")
def nuq():
    import paper_1908_06077_amd
    return paper_1908_06077_amd


def kind_of(nuq, name):
    return {"none": nuq.NO_NORM, "layer": nuq.LAYER_NORM, "rms": nuq.RMS_NORM}[name]


def rows_of(rows, hidden, kind, gen, pad=0, scale=1.0, shift=0.0):
    x = torch.randn(rows, hidden + pad, generator=gen, device=DEV) * scale + shift * torch.randn(rows, 1, generator=gen, device=DEV)
    return x.to(kind)[:, pad // 2:pad // 2 + hidden]


def close(got, want, bar, what=""):
    if got.numel():
        worst = float(((got.double() - want).abs() / bar).max())
        assert worst <= 1.0, (what, worst)


def rounded(value, bar, kind):
    """The bar of a value once it is rounded to its type."""
    return bar + HALF_UNIT[kind] * (1 + 4 * U) * (value.abs() + bar) + LEAST[kind]


def norm(s, name):
    """(n, mean, rstd, bar of n, of mean, of rstd) in fp64."""
    mean = s.mean(1, keepdim=True) if name == "layer" else torch.zeros_like(s[:, :1])
    top = s.abs().mean(1, keepdim=True) if name == "layer" else torch.zeros_like(mean)
    rstd = ((s - mean).square().mean(1, keepdim=True) + EPS).rsqrt()
    n = (s - mean) * rstd
    bar_mean = 66 * U * top + (2.0 ** -148 if name == "layer" else 0.0)
    off = 4 * (bar_mean * rstd) ** 2
    return n, mean, rstd, bar_mean * rstd + n.abs() * (40 * U + off), bar_mean, rstd * (36 * U + off)


def setting(rows, hidden, kind, weights, inner, outer, gen, pad, full):
    vector = lambda at: (at + 0.3 * torch.randn(hidden + 1, generator=gen, device=DEV)).to(weights)[1:].contiguous()  # noqa: E731
    v = {"w1": vector(1.0) if inner != "none" and full else None, "b1": vector(0.0) if inner != "none" and full else None,
         "gate": vector(0.4) if full else None, "w2": vector(1.0) if outer != "none" and full else None,
         "b2": vector(0.0) if outer != "none" and full else None}
    return v, rows_of(rows, hidden, kind, gen, pad, 2.0, 1.0), rows_of(rows, hidden, kind, gen, pad, 1.5, 0.5)


def forward(nuq, x, residual, v, inner, outer, numbers, total, y, stats):
    nuq.nuq_residual_norm_forward(x, residual, kind_of(nuq, inner), v["w1"], v["b1"], v["gate"], kind_of(nuq, outer), v["w2"], v["b2"],
                                  EPS, *numbers, total, y, stats)


@pytest.mark.parametrize("kind,weights", KINDS)
@pytest.mark.parametrize("rows,hidden", SHAPES)
def test_forward(nuq, rows, hidden, kind, weights):
    gen = torch.Generator(device=DEV).manual_seed(rows * 31 + hidden)
    for turn, (inner, outer) in enumerate(NORMS):
        pad, full, stream, p = ((0, True, True, 0.2), (3, True, True, 0.0), (5, False, True, 0.5), (0, True, False, 0.1))[turn % 4]
        scale, res = ((1.0, 1.0), (0.5, 0.7))[turn % 2]
        v, x, residual = setting(rows, hidden, kind, weights, inner, outer, gen, pad, full)
        residual = residual if stream else None
        wide = lambda: torch.full((rows, hidden + pad), 7.0, dtype=kind, device=DEV)  # noqa: E731
        total, y, stats = wide(), wide() if outer != "none" else None, torch.full((4, rows), 7.0, device=DEV)
        forward(nuq, x, residual, v, inner, outer, (scale, res, p, 77, None), total[:, :hidden], None if y is None else y[:, :hidden], stats)
        d = lambda t, other: other if t is None else t.double()  # noqa: E731
        b, bar = x.double(), torch.zeros(1, device=DEV, dtype=torch.float64)
        if inner != "none":
            b, mean, rstd, bar, bar_mean, bar_rstd = norm(b, inner)
            close(stats[1], rstd[:, 0], bar_rstd[:, 0], "rstd1")
            if inner == "layer":
                close(stats[0], mean[:, 0], bar_mean[:, 0], "mean1")
            w = d(v["w1"], 1.0)
            bar = bar * abs(w) + 2 * U * (b * w).abs() if v["w1"] is not None else bar
            b = b * w + d(v["b1"], 0.0)
            bar = bar + 2 * U * b.abs()
        f = scale * d(v["gate"], 1.0) * factors(rows, hidden, p, 77)
        r = residual.double() * res if stream else torch.zeros_like(b)
        s = b * f + r
        close(total[:, :hidden], s, rounded(s, bar * abs(f) + 5 * U * (b * f).abs() + 2 * U * r.abs() + U * s.abs(), kind), "total")
        assert (total[:, hidden:] == 7.0).all()
        if outer == "none":
            assert (stats[2:] == 7.0).all()
            continue
        n, mean, rstd, bar, bar_mean, bar_rstd = norm(total[:, :hidden].double(), outer)
        close(stats[3], rstd[:, 0], bar_rstd[:, 0], "rstd2")
        if outer == "layer":
            close(stats[2], mean[:, 0], bar_mean[:, 0], "mean2")
        else:
            assert (stats[2] == 7.0).all()
        w = d(v["w2"], 1.0)
        want = n * w + d(v["b2"], 0.0)
        close(y[:, :hidden], want, rounded(want, bar * abs(w) + 2 * U * (n * w).abs() + 2 * U * want.abs(), kind), "y")
        assert (y[:, hidden:] == 7.0).all()


def backward_formula(x, total, dy, dtotal, v, stats, inner, outer, numbers, f):
    """{name: (value, bar before rounding)} in fp64."""
    scale, res = numbers
    rows, hidden = x.shape
    m1, r1, m2, r2 = stats.double()[:, :, None]
    d = lambda t, other: torch.full((hidden,), other, dtype=torch.float64, device=DEV) if t is None else t.double()  # noqa: E731
    w1, b1, gate, w2 = d(v["w1"], 1.0), d(v["b1"], 0.0), d(v["gate"], 1.0), d(v["w2"], 1.0)
    many = (64 + rows / 256) * U
    out = {}
    mean = lambda t: t.mean(1, keepdim=True)  # noqa: E731

    def through(g, bar_g, n, rstd, name):
        s1, s2 = (mean(g) if name == "layer" else 0.0 * mean(g)), mean(g * n)
        bar1 = mean(bar_g) + 67 * U * mean(g.abs()) if name == "layer" else 0.0
        bar2 = mean(bar_g * n.abs()) + 70 * U * mean((g * n).abs())
        value = rstd * (g - s1 - n * s2)
        return value, rstd * (bar_g + bar1 + n.abs() * bar2 + 2 * U * g.abs() + 3 * U * s1.abs() + 6 * U * (n * s2).abs()) + 2 * U * value.abs()

    through_sum = dtotal.double() if dtotal is not None else torch.zeros_like(x, dtype=torch.float64)
    bar = torch.zeros_like(through_sum)
    if outer != "none":
        n = total.double()
        n = (n - m2 if outer == "layer" else n) * r2
        g = dy.double()
        out["dw2"] = ((g * n).sum(0), (g * n).abs().sum(0) * (many + 4 * U))
        out["db2"] = (g.sum(0), g.abs().sum(0) * many)
        value, bar = through(g * w2, U * (g * w2).abs(), n, r2, outer)
        through_sum = through_sum + value
        bar = bar + 2 * U * through_sum.abs()
    out["dresidual"] = (res * through_sum, abs(res) * bar + 2 * U * (res * through_sum).abs())
    g, bar = scale * f * through_sum, abs(scale) * f * bar + 4 * U * (scale * f * through_sum).abs()
    n = x.double()
    if inner != "none":
        n = (n - m1 if inner == "layer" else n) * r1
    whole = n * w1 + b1
    bar_whole = 5 * U * (n * w1).abs() + U * whole.abs()
    # dgate is w1 sum(g n) + b1 sum(g), so it is those magnitudes that round
    parts = (g * n * w1).abs() + (g * b1).abs()
    out["dgate"] = ((g * whole).sum(0), (bar * ((n * w1).abs() + b1.abs()) + g.abs() * bar_whole + 6 * U * parts).sum(0) + many * parts.sum(0))
    h, bar = g * gate, bar * gate.abs() + 3 * U * (g * gate).abs()
    out["dw1"] = ((h * n).sum(0), (bar * n.abs() + 6 * U * (h * n).abs()).sum(0) + many * (h * n).abs().sum(0))
    out["db1"] = (h.sum(0), bar.sum(0) + (many + 3 * U) * h.abs().sum(0))
    if inner != "none":
        h, bar = through(h * w1, bar * w1.abs() + U * (h * w1).abs(), n, r1, inner)
    out["dx"] = (h, bar)
    return out


GRADIENTS = (("dw1", "w1"), ("db1", "b1"), ("dgate", "gate"), ("dw2", "w2"), ("db2", "b2"))


def backward(nuq, dy, dtotal, x, total, v, inner, outer, numbers, stats, dx, dresidual, grads, ws):
    nuq.nuq_residual_norm_backward(dy, dtotal, x, total, kind_of(nuq, inner), v["w1"], v["b1"], v["gate"], kind_of(nuq, outer), v["w2"],
                                   *numbers, stats, dx, dresidual, *grads, ws)


def statistics(x, total, inner, outer):
    stats = torch.full((4, x.shape[0]), float("nan"), device=DEV)        # what a norm does not have is not read
    for k, (s, name) in enumerate(((x, inner), (total, outer))):
        if name != "none":
            _, mean, rstd, *_ = norm(s.double(), name)
            stats[2 * k + 1] = rstd[:, 0].float()
            if name == "layer":
                stats[2 * k] = mean[:, 0].float()
    return stats


@pytest.mark.parametrize("kind,weights", KINDS)
@pytest.mark.parametrize("rows,hidden", SHAPES)
def test_backward(nuq, rows, hidden, kind, weights):
    gen = torch.Generator(device=DEV).manual_seed(rows * 17 + hidden)
    ws = torch.empty(nuq.nuq_residual_norm_workspace_bytes(rows, hidden), dtype=torch.uint8, device=DEV)
    for turn, (inner, outer) in enumerate(NORMS):
        pad, full, through, p = ((0, True, True, 0.2), (3, True, True, 0.0), (5, False, True, 0.5), (0, True, False, 0.1))[turn % 4]
        scale, res = ((1.0, 1.0), (0.5, 0.7))[turn % 2]
        v, x, total = setting(rows, hidden, kind, weights, inner, outer, gen, pad, full)
        dy = rows_of(rows, hidden, kind, gen, pad, 0.5) if outer != "none" else None
        dtotal = rows_of(rows, hidden, kind, gen, pad, 0.5) if through or outer == "none" else None
        stats = statistics(x, total, inner, outer)
        wide = lambda: torch.full((rows, hidden + pad), 7.0, dtype=kind, device=DEV)  # noqa: E731
        dx, dresidual = wide(), wide()
        grads = [torch.empty_like(v[of]) if v[of] is not None else None for _, of in GRADIENTS]
        numbers = (scale, res, p, 78, None)
        backward(nuq, dy, dtotal, x, total if outer != "none" else None, v, inner, outer, numbers, stats, dx[:, :hidden],
                 dresidual[:, :hidden], grads, ws)
        want = backward_formula(x, total, dy, dtotal, v, stats, inner, outer, (scale, res), factors(rows, hidden, p, 78))
        for name, got in (("dx", dx[:, :hidden]), ("dresidual", dresidual[:, :hidden])):
            close(got, want[name][0], rounded(*want[name], kind), (name, inner, outer))
        for (name, _), got in zip(GRADIENTS, grads):
            if got is not None:
                close(got, want[name][0], rounded(*want[name], weights), (name, inner, outer))
        assert (dx[:, hidden:] == 7.0).all() and (dresidual[:, hidden:] == 7.0).all()
        if any(g is not None for g in grads):                # without the sums, and without the stream's gradient: the same rows
            again = torch.empty(rows, hidden, dtype=kind, device=DEV)
            backward(nuq, dy, dtotal, x, total if outer != "none" else None, v, inner, outer, numbers, stats, again, None, [None] * 5, None)
            assert torch.equal(again, dx[:, :hidden])


@pytest.mark.parametrize("rows,hidden", [(20_001, 40), (70_000, 9), (4097, 640), (9000, 2050), (3000, 5000), (2500, 9000)])
def test_sums_over_many_rows(nuq, rows, hidden):
    """Within their bar, and the same bits twice."""
    gen = torch.Generator(device=DEV).manual_seed(rows)
    v, x, total = setting(rows, hidden, BF16, F32, "layer", "layer", gen, 0, True)
    dy, dtotal = rows_of(rows, hidden, BF16, gen), rows_of(rows, hidden, BF16, gen)
    stats = statistics(x, total, "layer", "layer")
    ws = torch.empty(nuq.nuq_residual_norm_workspace_bytes(rows, hidden), dtype=torch.uint8, device=DEV)
    first = None
    for _ in range(2):
        dx, dresidual = torch.empty_like(x), torch.empty_like(x)
        grads = [torch.empty_like(v[of]) for _, of in GRADIENTS]
        backward(nuq, dy, dtotal, x, total, v, "layer", "layer", (1.0, 1.0, 0.1, 5, None), stats, dx, dresidual, grads, ws)
        ws.fill_(255)
        first = first or [dx, dresidual, *grads]
        assert all(torch.equal(a, b) for a, b in zip(first, [dx, dresidual, *grads]))
    want = backward_formula(x, total, dy, dtotal, v, stats, "layer", "layer", (1.0, 1.0), factors(rows, hidden, 0.1, 5))
    for (name, _), got in zip(GRADIENTS, grads):
        close(got, want[name][0], rounded(*want[name], F32), name)


def test_results_may_stand_where_the_rows_stood(nuq):
    gen = torch.Generator(device=DEV).manual_seed(8)
    for hidden in (5, 100, 1003, 1600, 4100, 8191, 16383):
        for inner, outer in NORMS:
            v, x, residual = setting(9, hidden, BF16, F32, inner, outer, gen, 0, True)
            numbers = (0.5, 0.7, 0.2, 3, None)
            new = lambda: torch.empty_like(x)  # noqa: E731
            total, y, stats = new(), new() if outer != "none" else None, torch.zeros(4, 9, device=DEV)
            forward(nuq, x, residual, v, inner, outer, numbers, total, y, stats)
            for at in (0, 1):                                # the sum in the place of either, the norm in the other's
                both = [x.clone(), residual.clone()]
                z = both[0] if at == 1 and y is not None else new()
                forward(nuq, both[0], both[1], v, inner, outer, numbers, both[at], z if y is not None else None, None)
                assert torch.equal(both[at], total) and (y is None or torch.equal(z, y))
            if hidden > 8192:                                # (the sums of wide rows are taken from what the results would replace)
                v = dict.fromkeys(v)
                forward(nuq, x, residual, v, inner, outer, numbers, total, y, stats)
            dy, dtotal = rows_of(9, hidden, BF16, gen) if y is not None else None, rows_of(9, hidden, BF16, gen)
            ws = torch.empty(nuq.nuq_residual_norm_workspace_bytes(9, hidden), dtype=torch.uint8, device=DEV)
            out = []
            for place in range(3):
                t = total.clone()
                grads = [torch.empty_like(v[of]) if v[of] is not None else None for _, of in GRADIENTS]
                g, a, xx = None if dy is None else dy.clone(), dtotal.clone(), x.clone()
                dx = (new(), g if g is not None else new(), xx)[place]
                dres = (new(), a, t if outer != "none" else a)[place]
                backward(nuq, g, a, xx, t if outer != "none" else None, v, inner, outer, numbers, stats, dx, dres, grads, ws)
                out.append([dx, dres, *[k for k in grads if k is not None]])
            for other in out[1:]:
                assert all(torch.equal(p, q) for p, q in zip(out[0], other)), (hidden, inner, outer)


def test_wide_rows_refuse_sums_in_place(nuq):
    v, x, residual = setting(3, 9000, BF16, F32, "layer", "layer", torch.Generator(device=DEV).manual_seed(1), 0, True)
    stats = statistics(x, residual, "layer", "layer")
    ws = torch.empty(nuq.nuq_residual_norm_workspace_bytes(3, 9000), dtype=torch.uint8, device=DEV)
    new = lambda: torch.empty_like(x)  # noqa: E731
    g, a, t = new().normal_(), new().normal_(), residual
    for dx, dres in ((g, new()), (x, new()), (new(), a), (new(), t)):
        with pytest.raises(nuq.NuqError, match="EINVAL"):
            backward(nuq, g, a, x, t, v, "layer", "layer", (1.0, 1.0, 0.0, 1, None), stats, dx, dres,
                     [torch.empty_like(v[of]) for _, of in GRADIENTS], ws)


def test_no_rows_and_missing_values(nuq):
    v, x, residual = setting(0, 33, F32, F32, "layer", "rms", torch.Generator(device=DEV).manual_seed(1), 0, True)
    stats = torch.empty(4, 0, device=DEV)
    forward(nuq, x, residual, v, "layer", "rms", (1.0, 1.0, 0.1, 1, None), torch.empty_like(x), torch.empty_like(x), stats)
    grads = [torch.full_like(v[of], 7.0) for _, of in GRADIENTS]
    backward(nuq, x, x, x, x, v, "layer", "rms", (1.0, 1.0, 0.1, 1, None), stats, torch.empty_like(x), None, grads,
             torch.empty(16, dtype=torch.uint8, device=DEV))
    assert not any(g.any() for g in grads)                   # sums over no rows
    gen = torch.Generator(device=DEV).manual_seed(4)
    for hidden in (40, 700, 9000):                           # what is not finite stays in its rows
        v, x, residual = setting(40, hidden, F32, F32, "layer", "layer", gen, 0, True)
        make = lambda: [torch.empty_like(x), torch.empty_like(x)]  # noqa: E731
        clean, got = make(), make()
        forward(nuq, x, residual, v, "layer", "layer", (1.0, 1.0, 0.0, 1, None), *clean, None)
        x[5, 3], x[9, hidden - 1], residual[20, 0] = float("nan"), float("inf"), -float("inf")
        forward(nuq, x, residual, v, "layer", "layer", (1.0, 1.0, 0.0, 1, None), *got, None)
        fine = [r for r in range(40) if r not in (5, 9, 20)]
        assert all(torch.equal(a[fine], b[fine]) for a, b in zip(clean, got)) and not got[1][[5, 9, 20]].isfinite().any()


def test_offsets_beyond_32_bits(nuq):
    hidden, stride, rows = 1001, (1 << 31) + 17, 3
    gen = torch.Generator(device=DEV).manual_seed(1)
    v, x, residual = setting(rows, hidden, BF16, F32, "layer", "layer", gen, 0, True)
    far = torch.zeros(stride * (rows - 1) + hidden, dtype=BF16, device=DEV).as_strided((rows, hidden), (stride, 1))
    numbers, stats = (1.0, 1.0, 0.1, 1, None), torch.empty(4, rows, device=DEV)
    new = lambda: torch.empty_like(x)  # noqa: E731
    want, got = (new(), new()), (new(), new())
    forward(nuq, x, residual, v, "layer", "layer", numbers, *want, stats)
    far.copy_(x)
    forward(nuq, far, residual, v, "layer", "layer", numbers, far, got[1], None)
    assert torch.equal(far, want[0]) and torch.equal(got[1], want[1])
    ws = torch.empty(nuq.nuq_residual_norm_workspace_bytes(rows, hidden), dtype=torch.uint8, device=DEV)
    grads = [[torch.empty_like(v[of]) for _, of in GRADIENTS] for _ in range(2)]
    backward(nuq, x, residual, x, want[0], v, "layer", "layer", numbers, stats, got[0], got[1], grads[0], ws)
    dres = new()
    backward(nuq, x, residual, x, far, v, "layer", "layer", numbers, stats, far, dres, grads[1], ws)
    assert torch.equal(far, got[0]) and torch.equal(dres, got[1]) and all(torch.equal(a, b) for a, b in zip(*grads))


# ---------------------------------------------------------------------------------------- the module

def module(hidden, weights=F32, **kw):
    from paper_1908_06077_amd.norm import ResidualNorm
    m = ResidualNorm(hidden, device=DEV, dtype=weights, **kw)
    gen = torch.Generator(device=DEV).manual_seed(hidden)
    for p in m.parameters():
        p.data.add_((0.2 * torch.randn(hidden, generator=gen, device=DEV)).to(weights))
    return m


@pytest.mark.parametrize("inner,outer", NORMS)
def test_module_gradients_against_differences(nuq, inner, outer):
    """Central differences of the formula in 64 bits, on a few elements of every input."""
    hidden, rows, h = 37, 6, 1e-5
    name = lambda k: None if k == "none" else k  # noqa: E731
    m = module(hidden, inner=name(inner), outer=name(outer), gate=0.5, scale=0.8, residual_scale=0.9, dropout=0.25, seed=9)
    gen = torch.Generator(device=DEV).manual_seed(2)
    x, r, gy, gt = (torch.randn(rows, hidden, generator=gen, device=DEV) for _ in range(4))
    x.requires_grad_()
    r.requires_grad_()
    seed = type(m.draws)(m.draws.p, m.draws.seed, None).next()
    out = m(x, r)
    y, total = out if outer != "none" else (None, out)
    ((total * gt).sum() + (0.0 if y is None else (y * gy).sum())).backward()
    f = factors(rows, hidden, 0.25, seed)

    def n(s, kind):
        s = s - s.mean(1, keepdim=True) if kind == "layer" else s
        return s * (s.square().mean(1, keepdim=True) + m.eps).rsqrt()

    def loss(x, r, w1, b1, gate, w2, b2):
        b = n(x, inner) * w1 + b1 if inner != "none" else x
        s = 0.9 * r + 0.8 * gate * b * f
        return float((s * gt.double()).sum() + (((n(s, outer) * w2 + b2) * gy.double()).sum() if outer != "none" else 0.0))
    params = [m.inner_weight, m.inner_bias, m.gate, m.outer_weight, m.outer_bias]
    inputs = [None if t is None else t.detach().double() for t in (x, r, *params)]
    for k, t in enumerate((x, r, *params)):
        if t is None:
            continue
        for at in range(0, t.numel(), 7):
            ends = []
            for sign in (1, -1):
                moved = [None if i is None else i.clone() for i in inputs]
                moved[k].view(-1)[at] += sign * h
                ends.append(loss(*moved))
            slope = (ends[0] - ends[1]) / (2 * h)            # error: h^2 times a third derivative of order ten, rounding 1e-13 / h
            assert abs(float(t.grad.view(-1)[at]) - slope) <= 1e-5 * (1.0 + abs(slope)), (k, at)


def test_module_accepts_what_autograd_hands_it(nuq):
    m = module(24, inner="rms", gate=0.3)
    gen = torch.Generator(device=DEV).manual_seed(5)
    x = torch.randn(24, 4, 3, generator=gen, device=DEV).permute(2, 1, 0).requires_grad_()     # rows that are not contiguous
    r = torch.randn(3, 4, 24, generator=gen, device=DEV, requires_grad=True)
    y, total = m(x, r)
    y.sum().backward()                                       # a gradient of stride zero, none through the sum
    assert y.shape == x.shape and x.grad.isfinite().all() and r.grad.isfinite().all()
    m.zero_grad()
    x.grad = r.grad = None
    m(x, r)[1].sum().backward()                              # the sum alone is used
    assert (r.grad == 1).all() and x.grad.isfinite().all() and not m.outer_weight.grad.any()
    frozen = module(24, inner="rms").requires_grad_(False)
    frozen(x, r.detach())[0].square().sum().backward()
    assert frozen.inner_weight.grad is None
    alone = module(24, inner=None, outer="rms", bias=False)
    assert alone(x)[0].shape == x.shape and alone.outer_bias is None      # no stream yet
    drop = module(24, dropout=0.5)
    a = drop(r, r)[1]
    assert not torch.equal(a, drop(r, r)[1])                 # every call draws anew
    drop.eval()
    assert torch.equal(drop(r, r)[1], drop(r, r)[1])
    from paper_1908_06077_amd.norm import ResidualNorm
    for bad in (lambda: m(torch.zeros(2, 25, device=DEV)), lambda: m(r, r[0]), lambda: ResidualNorm(20000),
                lambda: ResidualNorm(8, inner=None, outer=None), lambda: ResidualNorm(8, inner="batch"), lambda: ResidualNorm(8, dropout=2.0)):
        with pytest.raises(ValueError):
            bad()


def test_step_that_moves_between_forward_and_backward(nuq):
    """The backward pass repeats the mask of its own forward pass."""
    step = torch.zeros(1, dtype=torch.int64, device=DEV)
    m = module(64, inner="rms", outer=None, dropout=0.5, seed=4, step=step)
    x = torch.randn(50, 64, device=DEV, requires_grad=True)
    total = m(x, torch.zeros_like(x))
    step.fill_(9)
    total.backward(torch.ones_like(total))
    seed = type(m.draws)(0.5, 4, None).next()
    dropped = factors(50, 64, 0.5, seed) == 0
    assert torch.equal(total == 0, dropped)
    lone = torch.zeros_like(x)
    lone[3, int((~dropped[3]).nonzero()[0])] = 1.0
    assert x.grad.isfinite().all()


def test_forward_and_backward_replay_in_a_graph(nuq):
    for hidden in (1600, 9000):
        gen = torch.Generator(device=DEV).manual_seed(hidden)
        v, x, residual = setting(300, hidden, BF16, F32, "layer", "layer", gen, 0, True)
        step = torch.zeros(1, dtype=torch.int64, device=DEV)
        total, y, dx, dres, dy = (torch.empty_like(x) for _ in range(5))
        dy.normal_()
        stats = torch.zeros(4, 300, device=DEV)
        grads = [torch.empty_like(v[of]) for _, of in GRADIENTS]
        ws = torch.empty(nuq.nuq_residual_norm_workspace_bytes(300, hidden), dtype=torch.uint8, device=DEV)
        numbers = (1.0, 1.0, 0.3, 6, step)

        def both():
            forward(nuq, x, residual, v, "layer", "layer", numbers, total, y, stats)
            backward(nuq, dy, residual, x, total, v, "layer", "layer", numbers, stats, dx, dres, grads, ws)
        both()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            both()
        for k in range(4):
            x.normal_()
            step.fill_(k)
            both()
            out = (total, y, dx, dres, *grads)
            want = [t.clone() for t in out]
            for t in out:
                t.zero_()
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(want, out))


def test_another_stream(nuq):
    gen = torch.Generator(device=DEV).manual_seed(1)
    v, x, residual = setting(500, 1600, BF16, F32, "rms", "rms", gen, 0, True)
    want, got = [[torch.empty_like(x), torch.empty_like(x)] for _ in range(2)]
    numbers = (1.0, 1.0, 0.3, 6, None)
    forward(nuq, x, residual, v, "rms", "rms", numbers, *want, None)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        forward(nuq, x, residual, v, "rms", "rms", numbers, *got, None)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
