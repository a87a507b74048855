"""The gradients' norm of tensors that lie one behind the other, and of equal ones apart: other orders of summation, fp64 sums, so that
the rounded results differ by one unit of the last place of fp32 at most; and by nothing where the tensors are the same."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("sizes", [[3000, 3000], [1, 4095, 4097, 63], [100] * 400, [300_000, 5, 200_001], [8192 * 64] * 3])
def test_joined_and_apart(sizes, kind):
    import paper_1908_06077_amd as nuq
    ws = torch.empty(nuq.GRADIENT_NORM_WORKSPACE_BYTES, dtype=torch.uint8, device=DEV)
    for seed in range(20):
        gen = torch.Generator(device=DEV).manual_seed(seed)
        flat = torch.randn(sum(sizes), generator=gen, device=DEV).to(kind)
        joined = list(flat.split(sizes))
        apart = [x.clone() for x in reversed(joined)][::-1]
        out = torch.empty(3, 2, device=DEV)
        for k, tensors in enumerate((joined, apart, joined)):
            nuq.nuq_gradient_norm(tensors, 0.5, ws, out[k])
        assert torch.equal(out[0], out[2])
        exact = float(flat.double().square().sum().sqrt())
        for norm, factor in out.tolist():
            assert abs(norm - exact) <= 2.0 ** -24 * 1.01 * exact and abs(factor - 0.5 / exact) <= 2.0 ** -24 * 1.01 * factor
        assert torch.all((out[0] - out[1]).abs() <= 2.0 ** -23 * out[0])
