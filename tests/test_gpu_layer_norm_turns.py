"""Layer norm of more rows than the device's teams hold at once: every team takes several, each loaded while the one before is
worked on.  Formulas and bars are those of test_gpu_layer_norm.py; weight gradients lose at most 64 + rows / 256 roundings."""
import pytest
import torch

from test_gpu_layer_norm import BF16, DEV, F16, F32, HALF_UNIT, LEAST, U, close, forward_formula, rows_of

pytestmark = pytest.mark.gpu

KINDS = [(F32, F32), (BF16, F32), (F16, F16)]
# more than three times 8 workgroups per CU of 256 threads; two to eight times 512 workgroups
FORWARD = [(400_000, 7), (400_000, 31), (100_000, 40), (100_001, 200), (50_000, 512), (25_000, 1001), (13_000, 1600), (7_000, 4095),
           (3_500, 8192), (2_600, 12_287), (1_600, 16_384)]
BACKWARD = [(400_000, 7), (300_000, 31), (100_000, 100), (40_001, 200), (25_000, 512), (12_001, 1000), (9_000, 1600), (4_500, 4095),
            (3_000, 8192), (1_500, 12_287), (1_500, 16_384)]


@pytest.fixture(scope="module")
def nuq():
    import paper_1908_06077_amd
    return paper_1908_06077_amd


@pytest.mark.parametrize("kind,weights", KINDS)
@pytest.mark.parametrize("rows,hidden", FORWARD)
def test_forward(nuq, rows, hidden, kind, weights):
    gen = torch.Generator(device=DEV).manual_seed(rows + hidden)
    weight, bias = ((at + 0.3 * torch.randn(hidden, generator=gen, device=DEV)).to(weights) for at in (1.0, 0.0))
    x, r = rows_of(rows, hidden, kind, gen, 0, 2.0, 3.0), rows_of(rows, hidden, kind, gen)
    mean, rstd = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    for stream in (False, True):
        s = (x.float() + r.float()).to(kind) if stream else x
        want = forward_formula(s, weight, bias, 1e-5, kind)
        for place in ("apart", "x", "residual")[:3 if stream else 2]:          # where the results stand
            a, b, y = x.clone(), r.clone(), torch.empty_like(x)
            total = {"apart": torch.empty_like(x), "x": a, "residual": b}[place] if stream else None
            if place == "x" and not stream:
                y = a
            mean.fill_(7.0)
            rstd.fill_(7.0)
            nuq.nuq_layer_norm_forward(a, b if stream else None, weight, bias, 1e-5, total, y, mean, rstd)
            close(y, want[0], want[3])
            close(mean, want[1], want[4])
            close(rstd, want[2], want[5])
            assert total is None or torch.equal(total, s)


@pytest.mark.parametrize("kind,weights", KINDS)
@pytest.mark.parametrize("rows,hidden", BACKWARD)
def test_backward(nuq, rows, hidden, kind, weights):
    gen = torch.Generator(device=DEV).manual_seed(rows + hidden)
    x, dy, add = (rows_of(rows, hidden, kind, gen, 0, *k) for k in ((2.0, 3.0), (0.5,), (1.0,)))
    weight = (1.0 + 0.3 * torch.randn(hidden, generator=gen, device=DEV)).to(weights)
    s = x.double()
    mean = s.mean(1).float()
    rstd = (s.var(1, correction=0) + 1e-5).rsqrt().float()
    r = rstd.double()[:, None]
    n, d = (s - mean.double()[:, None]) * r, dy.double()
    many = (64 + rows / 256) * U
    dn = d * n
    want_w, bar_w, want_b, bar_b = dn.sum(0), dn.abs().sum(0) * (many + 4 * U), d.sum(0), d.abs().sum(0) * many
    d = d * weight.double()
    dn = d * n
    s1, s2, a1, a2 = d.mean(1, keepdim=True), dn.mean(1, keepdim=True), d.abs().mean(1, keepdim=True), dn.abs().mean(1, keepdim=True)
    plain = r * (d - s1 - n * s2)
    bar = r * (68 * U * (a1 + n.abs() * a2) + 8 * U * (d.abs() + s1.abs() + (n * s2).abs()))
    del s, d, dn
    ws = torch.empty(nuq.nuq_layer_norm_workspace_bytes(rows, hidden), dtype=torch.uint8, device=DEV)
    for plus in (None, add):
        want = plain if plus is None else plain + plus.double()
        bar_x = bar + U * want.abs() + HALF_UNIT[kind] * (want.abs() + bar) + LEAST[kind]
        for in_place in (False, True):
            g = dy.clone()
            dx = g if in_place else torch.empty_like(g)
            dw, db = (torch.full((hidden,), 7.0, dtype=weights, device=DEV) for _ in range(2))
            nuq.nuq_layer_norm_backward(g, x, weight, mean, rstd, plus, dx, dw, db, ws)
            close(dx, want, bar_x)
            close(dw, want_w, bar_w + want_w.abs() * HALF_UNIT[weights] + LEAST[weights])
            close(db, want_b, bar_b + want_b.abs() * HALF_UNIT[weights] + LEAST[weights])
            g = dy.clone()
            again = g if in_place else torch.empty_like(g)
            nuq.nuq_layer_norm_backward(g, x, weight, mean, rstd, plus, again, None, None, None)
            assert torch.equal(again, dx)                    # without the sums: other launches, the same rows


def test_more_long_rows_than_a_launch_has_workgroups(nuq):
    """2^21 workgroups at most; rows that overlap in memory stand in for as many of their own."""
    rows, hidden = (1 << 21) + 300, 16_385
    gen = torch.Generator(device=DEV).manual_seed(1)
    flat = torch.randn(rows * 8 + hidden, generator=gen, device=DEV).to(BF16)
    x = flat.as_strided((rows, hidden), (8, 1))
    y = torch.zeros(rows, hidden, dtype=BF16, device=DEV)
    stats, few = torch.zeros(2, rows, device=DEV), torch.zeros(2, 300, device=DEV)
    nuq.nuq_layer_norm_forward(x, None, None, None, 1e-5, None, y, stats[0], stats[1])
    want = torch.empty(300, hidden, dtype=BF16, device=DEV)
    for first in (0, (1 << 21) - 300, rows - 300):
        nuq.nuq_layer_norm_forward(x[first:first + 300], None, None, None, 1e-5, None, want, few[0], few[1])
        assert torch.equal(y[first:first + 300], want) and torch.equal(stats[:, first:first + 300], few)
    nuq.nuq_layer_norm_backward(x, x, None, stats[0], stats[1], None, y, None, None, None)
    for first in (0, (1 << 21) - 300, rows - 300):
        nuq.nuq_layer_norm_backward(x[first:first + 300], x[first:first + 300], None, stats[0][first:first + 300],
                                    stats[1][first:first + 300], None, want, None, None, None)
        assert torch.equal(y[first:first + 300], want)
