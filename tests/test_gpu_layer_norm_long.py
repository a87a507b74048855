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
