"""AdamW where its numbers are extreme: second moments below the least normal float, and eps at both ends of what is accepted.

Bars (u = 2^-24): 32 u of the update, of which 16 are its own roundings and 16 those of m, v and the constants; a v that is subnormal
is held to 2^-149 (three such roundings), half of which, relative to v, the root takes over."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")
U = 2.0 ** -24


def one_step(coded, w, g, alpha, beta1, beta2, eps):
    import paper_1908_06077_amd as nuq
    n = w.numel()
    if coded:
        m = torch.zeros(n, dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn)
        v, scales = torch.zeros(n, dtype=torch.uint8, device=DEV), torch.zeros(2 * nuq.nuq_state_blocks(n), device=DEV)
        nuq.nuq_adamw_step_coded([w], [g], [m], [v], [scales], None, alpha, beta1, beta2, eps, 1)
    else:
        nuq.nuq_adamw_step([w], [g], [torch.zeros_like(w)], [torch.zeros_like(w)], None, alpha, beta1, beta2, eps, 1)
    assert nuq.nuq_last_error_flags() == 0


def check(coded, g, alpha, beta1, beta2, eps):
    """A first step from weights and states of zero: the weights are the update alone."""
    w = torch.zeros(g.size, device=DEV)
    one_step(coded, w, torch.from_numpy(g).to(DEV), alpha, beta1, beta2, eps)
    f = np.float64
    m, v = (1.0 - beta1) * g.astype(f), (1.0 - beta2) * g.astype(f) ** 2
    want = -alpha / (1.0 - beta1) * m / (np.sqrt(v) / np.sqrt(1.0 - beta2) + eps)
    root = np.sqrt(v) / (np.sqrt(v) + eps * np.sqrt(1.0 - beta2))            # the root's share of the denominator
    bar = np.abs(want) * (32 * U + root * 2.0 ** -149 / np.maximum(v, 2.0 ** -149) * 1.5) + 2.0 ** -140
    worst = np.max(np.abs(w.cpu().numpy().astype(f) - want) / bar)
    assert worst <= 1.0, (worst, w[:8].tolist(), want[:8])


@pytest.mark.parametrize("coded", [False, True])
@pytest.mark.parametrize("eps", [1e-30, 1e-37, 1e-20])
def test_second_moments_below_the_least_normal_float(coded, eps):
    """v from 1.6e-41, some ten thousand times the least subnormal, through 1e-38 to 1e-36."""
    g = np.concatenate([np.geomspace(4e-20, 1e-17, 300), -np.geomspace(4e-20, 1e-17, 300)]).astype(np.float32)
    check(coded, g, 1e-3, 0.9, 0.99, eps)


@pytest.mark.parametrize("coded", [False, True])
@pytest.mark.parametrize("eps", [1e10, 1e25, 8e37, 3e38])
def test_an_eps_above_every_second_moment(coded, eps):
    """The denominator's reciprocal passes below the least normal float."""
    g = np.geomspace(1.0, 1e18, 700).astype(np.float32)
    check(coded, g, 1e30, 0.9, 0.99, eps)
