"""AdamW with states in 8 bits where a step moves the moments by less than a code holds: codes that are drawn, exactly, and moments
that follow the gradients all the same.

Bars.  A code's steps are 1/16 to 1/8 of its value, 0.087 in the mean over a logarithmic spread.  A step moves v against its block's
scale by (1 - beta2) |x - y| of itself, x and y squares of normal numbers, 1.3 in the mean; a draw adds 0.087 times that to the
variance, which beta2 forgets at a rate of 2 (1 - beta2): 0.056 in all, a standard deviation of 0.24 for v and of 0.12 for its
root.  A median of N such roots is known to 1.25 * 0.12 / sqrt(N), and lies below 1 by an eighth of the variance and its skew."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")


@pytest.fixture(scope="module")
def nuq():
    import paper_1908_06077_amd
    return paper_1908_06077_amd


class State:
    """Weights, and moments in codes or in fp32."""

    def __init__(self, nuq, n, coded):
        self.nuq, self.coded, self.n = nuq, coded, n
        self.w = torch.zeros(n, device=DEV)
        if coded:
            self.m = torch.zeros(n, dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn)
            self.v = torch.zeros(n, dtype=torch.uint8, device=DEV)
            self.scales = torch.zeros(2 * nuq.nuq_state_blocks(n), device=DEV)
        else:
            self.m, self.v = torch.zeros(n, device=DEV), torch.zeros(n, device=DEV)

    def step(self, g, t, beta1=0.9, beta2=0.999, alpha=1e-3):
        if self.coded:
            self.nuq.nuq_adamw_step_coded([self.w], [g], [self.m], [self.v], [self.scales], None, alpha, beta1, beta2, 1e-8, t)
        else:
            self.nuq.nuq_adamw_step([self.w], [g], [self.m], [self.v], None, alpha, beta1, beta2, 1e-8, t)

    def moments(self):
        if not self.coded:
            return self.m.clone(), self.v.clone()
        m, v = torch.empty(self.n, device=DEV), torch.empty(self.n, device=DEV)
        self.nuq.nuq_adamw_state_values(self.m, self.v, self.scales, m, v)
        return m, v


# ---------------------------------------------------------------------------------------- codes, exactly

def bits(x):
    return np.ascontiguousarray(x, dtype=np.float32).view(np.uint32)


def drawn_codes(m, v, t, draw_m, draw_v):
    """Codes and scales of moments of whole blocks, from the definition in the header; uint32 arithmetic wraps."""
    u, uu, f = np.uint32, np.uint64, np.float32
    m, v = m.reshape(-1, 256), v.reshape(-1, 256)
    a, e = np.abs(m).max(1, keepdims=True), v.max(1, keepdims=True)
    a[a < 2.0 ** -126], e[e < 2.0 ** -126] = 0.0, 0.0
    with np.errstate(divide="ignore"):
        ia, ie = np.where(a > 0, f(1) / a, f(0)).astype(f), np.where(e > 0, f(1) / e, f(0)).astype(f)
    z = (bits(a).astype(uu) << uu(32) | bits(e).astype(uu)) + uu(t * 0x9E3779B97F4A7C15 & (1 << 64) - 1)
    z = (z ^ z >> uu(30)) * uu(0xBF58476D1CE4E5B9)
    z = (z ^ z >> uu(27)) * uu(0x94D049BB133111EB)
    z ^= z >> uu(31)
    x = ((z & uu(0xFFFFFFFF)).astype(u) + np.arange(256, dtype=u)) * u(0x9E3779B1)
    x = (x ^ x >> u(15) ^ (z >> uu(32)).astype(u)) * u(0x85EBCA6B)
    x ^= x >> u(16)
    y = x * u(0x9E3779B1)
    y ^= y >> u(15)
    below = lambda b, r, drawn: ((r >> u(12) & u(0xFFFF0)) | u(8)) if drawn else u(0x7FFFF) + (b >> u(20) & u(1))  # noqa: E731
    bv = bits(v * ie * f(2.0 ** -96))
    cv = np.maximum((bv + below(bv, x, draw_v)) >> u(20), ((v > 0) & (e > 0)).astype(u))
    bm = bits(m * ia * f(2.0 ** -112))
    cm = ((bm & u(0x7FFFFFFF)) + below(bm & u(0x7FFFFFFF), y, draw_m)) >> u(20) | (bm >> u(24) & u(0x80))
    return cm.astype(np.uint8).reshape(-1), cv.astype(np.uint8).reshape(-1), np.concatenate([a, e], 1).reshape(-1)


@pytest.mark.parametrize("beta1,beta2,t", [(0.9, 0.999, 16), (0.9, 0.999, 17), (0.97, 0.999, 1000), (0.99, 0.95, 10 ** 6),
                                           (0.95, 0.9, 2 ** 40 + 1), (0.0, 0.9999, 500), (0.9, 0.95, 30)])
@pytest.mark.parametrize("grad", [torch.float32, torch.bfloat16])
def test_codes(nuq, beta1, beta2, t, grad):
    rng = np.random.default_rng(t)
    n, f = 256 * 37, np.float32
    scale = np.repeat(10.0 ** rng.uniform(-9, 3, 37), 256) * 10.0 ** rng.uniform(-3, 0, n)
    s = State(nuq, n, True)
    for k in range(4):                                       # (the later ones from codes that were drawn)
        g = torch.from_numpy((rng.standard_normal(n) * scale * (rng.random(n) < 0.8)).astype(f)).to(DEV).to(grad)
        m, v = (x.cpu().numpy() for x in s.moments())
        s.step(g, t + k, beta1, beta2)
        g = g.float().cpu().numpy()
        m, v = m * f(beta1) + g * f(1.0 - beta1), v * f(beta2) + g * g * f(1.0 - beta2)
        share = [(1.0 - b) / -np.expm1((t + k) * np.log(b)) if b else 1.0 for b in (beta1, beta2)]
        cm, cv, scales = drawn_codes(m, v, t + k, share[0] < 1 / 16, share[1] < 1 / 16)
        np.testing.assert_array_equal(s.scales.cpu().numpy(), scales)
        np.testing.assert_array_equal(s.v.cpu().numpy(), cv)
        np.testing.assert_array_equal(s.m.view(torch.uint8).cpu().numpy(), cm)
    assert nuq.nuq_last_error_flags() == 0


def test_the_same_bits_joined_and_apart_and_in_short_blocks(nuq):
    """Tensors that follow each other in memory and the same elsewhere: a draw does not depend on where a tensor stands."""
    gen = torch.Generator(device=DEV).manual_seed(1)
    sizes = [256, 1024, 77]
    g = [torch.randn(n, generator=gen, device=DEV) for n in sizes]
    whole = State(nuq, sum(sizes), True)
    apart = [State(nuq, n, True) for n in sizes]
    split = lambda x: list(x.split(sizes))  # noqa: E731
    scales = list(whole.scales.split([2 * nuq.nuq_state_blocks(n) for n in sizes]))
    for t in (1000, 1001, 1002):
        nuq.nuq_adamw_step_coded(split(whole.w), g, split(whole.m), split(whole.v), scales, None, 1e-3, 0.95, 0.999, 1e-8, t)
        nuq.nuq_adamw_step_coded([s.w for s in apart], [x.clone() for x in g], [s.m for s in apart], [s.v for s in apart],
                                 [s.scales for s in apart], None, 1e-3, 0.95, 0.999, 1e-8, t)
    for a, b in zip(apart, range(3)):
        assert torch.equal(a.w, split(whole.w)[b]) and torch.equal(a.v, split(whole.v)[b]) and torch.equal(a.scales, scales[b])
        assert torch.equal(a.m.view(torch.uint8), split(whole.m.view(torch.uint8))[b])


def test_zero_gradients_fade_a_whole_block_without_loss(nuq):
    """Values on their codes stay there while the scale shrinks, drawn or not: after 500 steps every ratio is as it was."""
    n = 256 * 8
    gen = torch.Generator(device=DEV).manual_seed(4)
    s = State(nuq, n, True)
    s.step(torch.randn(n, generator=gen, device=DEV), 1, beta1=0.97)
    before = s.m.view(torch.uint8).clone(), s.v.clone()
    for t in range(1000, 1500):
        s.step(torch.zeros(n, device=DEV), t, beta1=0.97)
    assert torch.equal(s.m.view(torch.uint8), before[0]) and torch.equal(s.v, before[1])


# ---------------------------------------------------------------------------------------- moments that follow

def roots(coded, plain):
    return (coded.moments()[1] / plain.moments()[1]).sqrt()


@pytest.mark.parametrize("change", [1.0, 4.0, 0.25])
def test_v_follows_gradients_at_the_default_beta2(nuq, change):
    """4000 steps of gradients of one size each (over one decade), then 4000 in which one in sixteen is `change` times as large."""
    n = 1 << 16
    gen = torch.Generator(device=DEV).manual_seed(7)
    size = 10.0 ** -torch.rand(n, generator=gen, device=DEV)
    coded, plain = State(nuq, n, True), State(nuq, n, False)
    for t in range(1, 8001):
        if t == 4001:
            size[::16] *= change
        g = torch.randn(n, generator=gen, device=DEV) * size
        coded.step(g, t)
        plain.step(g, t)
        if t in (4000, 8000):
            r = roots(coded, plain)
            one = torch.arange(n, device=DEV) % 16 == 0
            for part in (r[one], r[~one]):
                low, middle, high = torch.quantile(part, torch.tensor([0.01, 0.5, 0.99], device=DEV)).tolist()
                assert 0.95 < middle < 1.02, (t, middle)
                # three standard deviations; v that shrinks still holds 1.8 % of what was 16 times as large, drawn by its steps
                assert low > 0.64 and high < (1.36 if t == 4000 or change >= 1.0 else 1.6), (t, low, high)
    assert nuq.nuq_last_error_flags() == 0


@pytest.mark.parametrize("beta1,beta2", [(0.9, 0.999), (0.99, 0.999), (0.97, 0.95)])
def test_moments_whose_gradients_end_fade_in_the_mean(nuq, beta1, beta2):
    """Half of every block sees no more gradients beside a half that does; steps from a millionth on, so that all codes of betas above
    15/16 are drawn.  The mean of v, and of |m|, over the N of them against fp32: each ratio has a standard deviation below 1
    while it is above a hundredth of the others, so 5 / sqrt(N), and a draw keeps the mean to 2^-16 of a step."""
    n, steps, begin = 1 << 16, int(1.0 / (1.0 - max(beta1, beta2))), 10 ** 6
    gen = torch.Generator(device=DEV).manual_seed(9)
    coded, plain = State(nuq, n, True), State(nuq, n, False)
    quiet = torch.arange(n, device=DEV) % 2 == 0
    sign = torch.where(torch.rand(n, generator=gen, device=DEV) < 0.5, -1.0, 1.0)
    looked = 0
    for k in range(1, 2 * steps + 1):
        g = sign * (1.0 + 0.1 * torch.randn(n, generator=gen, device=DEV))     # of one sign, so that m is large too
        if k > steps:
            g[quiet] = 0.0
        coded.step(g, begin + k, beta1, beta2)
        plain.step(g, begin + k, beta1, beta2)
        if k in (steps, steps + 20, 2 * steps):
            (m, v), (pm, pv) = coded.moments(), plain.moments()
            for x, y, beta in ((m.abs(), pm.abs(), beta1), (v, pv, beta2)):
                if beta > 15 / 16 and float(y[quiet].mean()) > 0.01 * float(y[~quiet].mean()):
                    looked += 1
                    assert abs(float((x / y)[quiet].mean()) - 1.0) < 5.0 / (n / 2) ** 0.5 + 0.002, (k, beta)
    assert looked >= 3


def test_a_noisy_quadratic_ends_as_low_as_with_fp32_at_the_default_betas(nuq):
    """Steps that are 12 % uneven cost the end about 1 %; the bar is ten times that.  (Nearest codes throughout: 19 % more.)"""
    n, far = 1 << 14, {}
    for is_coded in (False, True):
        gen = torch.Generator(device=DEV).manual_seed(1)
        target = torch.randn(n, generator=gen, device=DEV)
        curve = 10.0 ** torch.empty(n, device=DEV).uniform_(-1, 1, generator=gen)
        s = State(nuq, n, is_coded)
        for t in range(1, 4001):
            s.step(curve * (s.w - target + 0.1 * torch.randn(n, generator=gen, device=DEV)), t, alpha=1e-2 * (1.0 - t / 4001))
        far[is_coded] = float((s.w - target).square().mean().sqrt())
    assert far[True] < 1.1 * far[False], far
