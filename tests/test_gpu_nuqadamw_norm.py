"""What NUQAdamW.norm holds before a norm was taken: NaN, not what the memory held."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")


@pytest.mark.parametrize("max_norm", [None, 1.0])
def test_norm_before_and_behind_steps(max_norm):
    from paper_1908_06077_amd.optim import NUQAdamW
    held = torch.full((2,), 3.0, device=DEV)                 # (the allocator hands this memory out again)
    del held
    p = torch.nn.Parameter(torch.ones(300, device=DEV))
    opt = NUQAdamW([p], K=1, lr=0.1, bucket=128, s=4, max_norm=max_norm)
    assert torch.isnan(opt.norm).all()
    with opt.worker(0):
        p.sum().backward()
    opt.step()
    assert torch.isnan(opt.norm).all() if max_norm is None else torch.isfinite(opt.norm).all()
