"""The residual norm's results in the place of the rows they are of, in teams of more than a wave and rows that are not whole vectors: a
column is then two threads', of two waves, and what one stores must not be there before the other has read."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")


@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("hidden", [515, 1001, 1603, 2051, 4100, 6001, 8191])
def test_gradient_in_the_place_of_the_branch(kind, hidden):
    """No norm of the branch: x enters the gate's gradient alone, and its gradient is stored behind a single barrier.  The same bits as with
    a place of its own, whatever the rows per team."""
    import paper_1908_06077_amd as nuq
    gen = torch.Generator(device=DEV).manual_seed(hidden)
    rows = 4001
    x, total, dy, dtotal = (torch.randn(rows, hidden, generator=gen, device=DEV).to(kind) for _ in range(4))
    gate, w2 = (1.0 + 0.2 * torch.randn(hidden, generator=gen, device=DEV) for _ in range(2))
    ws = torch.empty(nuq.nuq_residual_norm_workspace_bytes(rows, hidden), dtype=torch.uint8, device=DEV)
    for outer in (nuq.LAYER_NORM, nuq.RMS_NORM):
        stats = torch.empty(4, rows, device=DEV)
        y = torch.empty_like(x)
        nuq.nuq_residual_norm_forward(x, total, nuq.NO_NORM, None, None, gate, outer, w2, None, 1e-5, 1.0, 1.0, 0.1, 7, None, y, y.clone(), stats)
        want = None
        for place in (torch.empty_like(x), x.clone(), x.clone(), x.clone()):
            own = place if want is not None else x
            dresidual, dgate, dw2 = torch.empty_like(x), torch.empty_like(gate), torch.empty_like(w2)
            nuq.nuq_residual_norm_backward(dy, dtotal, own, y, nuq.NO_NORM, None, None, gate, outer, w2, 1.0, 1.0, 0.1, 7, None, stats, place,
                                           dresidual, None, None, dgate, dw2, None, ws)
            got = (place, dresidual, dgate, dw2)
            want = want or got
            assert all(torch.equal(a, b) for a, b in zip(want, got)), outer
