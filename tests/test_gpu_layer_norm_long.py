"""Layer norm of rows so long that launches and sums meet their limits."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")
U = 2.0 ** -24


@pytest.fixture(scope="module")
def nuq():
    import paper_1908_06077_amd
    return paper_1908_06077_amd


@pytest.mark.parametrize("rows", [0, 1, 2])
def test_weight_gradients_of_more_columns_than_a_launch_has_workgroups_for(nuq, rows):
    """2^26 + 21 columns; statistics that make every product and sum of two rows exact to one rounding."""
    hidden = (1 << 26) + 21
    gen = torch.Generator(device=DEV).manual_seed(rows)
    x, dy = torch.randn(rows, hidden, generator=gen, device=DEV), torch.randn(rows, hidden, generator=gen, device=DEV)
    mean, rstd = torch.full((rows,), 0.5, device=DEV), torch.full((rows,), 2.0, device=DEV)
    dw, db = torch.full((hidden,), 7.0, device=DEV), torch.full((hidden,), 7.0, device=DEV)
    ws = torch.empty(max(16, nuq.nuq_layer_norm_workspace_bytes(rows, hidden)), dtype=torch.uint8, device=DEV)
    dx = torch.empty_like(x)
    nuq.nuq_layer_norm_backward(dy, x, None, mean, rstd, None, dx, dw, db, ws)
    n = (x - 0.5) * 2.0
    assert torch.equal(db, dy.sum(0) if rows else torch.zeros_like(db))
    assert torch.equal(dw, (dy * n).sum(0) if rows else torch.zeros_like(dw))


# Bars of sums over long rows: at most eight elements of a vector are added in fp32, vectors in fp64, then six steps over a wave and
# sixteen waves: 32 u of the mean magnitude, whatever the length.

def close(got, want, bar):
    worst = float(((got.double() - want).abs() / bar).max())
    assert worst <= 1.0, worst


@pytest.mark.parametrize("hidden", [16_385, 5_000_003, 40_000_000])
def test_statistics_of_long_rows_far_from_zero(nuq, hidden):
    """A mean a hundred times the spread: what the row's sums lose shows in every element."""
    gen = torch.Generator(device=DEV).manual_seed(hidden)
    x = 0.1 + 1e-3 * torch.randn(2, hidden, generator=gen, device=DEV)
    r = torch.zeros_like(x)
    s = x.double()
    mean = s.mean(1)
    rstd = 1.0 / (s - mean[:, None]).square().mean(1).sqrt()
    bar_mean = 33 * U * s.abs().mean(1)
    bar_rstd = rstd * (20 * U + 4 * (bar_mean * rstd) ** 2)
    n = (s - mean[:, None]) * rstd[:, None]
    bar_n = (bar_mean * rstd)[:, None] + n.abs() * (24 * U + 4 * ((bar_mean * rstd) ** 2)[:, None]) + U * n.abs()
    for residual in (None, r):
        y, total, m, q = torch.empty_like(x), torch.empty_like(x), torch.empty(2, device=DEV), torch.empty(2, device=DEV)
        nuq.nuq_layer_norm_forward(x, residual, None, None, 0.0, None if residual is None else total, y, m, q)
        close(m, mean, bar_mean)
        close(q, rstd, bar_rstd)
        close(y, n, bar_n)


@pytest.mark.parametrize("hidden", [16_385, 5_000_003, 40_000_000])
def test_gradients_of_long_rows_far_from_zero(nuq, hidden):
    gen = torch.Generator(device=DEV).manual_seed(hidden)
    x, dy = torch.randn(2, hidden, generator=gen, device=DEV), 0.1 + 1e-3 * torch.randn(2, hidden, generator=gen, device=DEV)
    x = x + 1.0
    mean, rstd = torch.full((2,), 0.3, device=DEV), torch.full((2,), 0.7, device=DEV)    # any statistics: n is far from zero too
    dx = torch.empty_like(x)
    nuq.nuq_layer_norm_backward(dy, x, None, mean, rstd, None, dx, None, None, None)
    d, n, q = dy.double(), (x.double() - mean.double()[:, None]) * rstd.double()[:, None], rstd.double()[:, None]
    s1, s2 = d.mean(1, keepdim=True), (d * n).mean(1, keepdim=True)
    a2 = (d * n).abs().mean(1, keepdim=True)
    bar = q * (36 * U * (s1.abs() + n.abs() * a2) + 8 * U * (d.abs() + s1.abs() + (n * s2).abs()))
    want = q * (d - s1 - n * s2)
    close(dx, want, bar + U * want.abs())


def test_weight_gradients_of_many_long_rows(nuq):
    """60 000 rows whose gradients repeat, so that an addition's rounding repeats too.  64 groups of rows, each in pieces of 32 rows:
    32 + rows / 2048 additions, then 20 that add up the groups."""
    rows, hidden = 60_000, 16_400
    gen = torch.Generator(device=DEV).manual_seed(3)
    line = 0.05 + 0.1 * torch.rand(hidden, generator=gen, device=DEV)
    x, dy = torch.full((rows, hidden), 1.5, device=DEV), line.expand(rows, hidden).contiguous()
    mean, rstd = torch.full((rows,), 0.5, device=DEV), torch.ones(rows, device=DEV)      # n = 1
    dw, db = torch.empty(hidden, device=DEV), torch.empty(hidden, device=DEV)
    ws = torch.empty(nuq.nuq_layer_norm_workspace_bytes(rows, hidden), dtype=torch.uint8, device=DEV)
    nuq.nuq_layer_norm_backward(dy, x, None, mean, rstd, None, torch.empty_like(x), dw, db, ws)
    want = rows * line.double()
    for got in (dw, db):
        close(got, want, want * U * (52 + rows / 2048 + 2))
