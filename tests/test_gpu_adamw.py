"""AdamW on lists of tensors and the gradients' norm against their formulas in 64 bits.

Bars.  u = 2^-24 is half a unit of the last place of fp32.  m: three constants and products rounded, one sum: at most 4 u of the
summed magnitudes, one more behind a coefficient; v: two more for g * g.  w: its own two products and sum, 4 u of |w|; the update
inherits m's error, half of v's, and takes a square root and a reciprocal of one unit each, two products and the rounded
constants: 16 u of itself.  8-bit states: codes and scales have to be those of the fp32 formula with the nearest representable
value found by search, exactly."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")
U = 2.0 ** -24
HYPER = dict(alpha=1e-2, beta1=0.9, beta2=0.99, eps=1e-8, t=3)
TYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def nuq():
    import paper_1908_06077_amd
    return paper_1908_06077_amd


def to_dev(a, dtype=torch.float32, shift=0):
    """A device tensor of a's values that begins `shift` elements behind an allocation's begin."""
    t = torch.empty(a.size + shift, dtype=dtype, device=DEV)[shift:]
    t.copy_(torch.from_numpy(np.ascontiguousarray(a)))
    return t


def vectors(n, rng):
    scale = 10.0 ** rng.uniform(-6, 1, n)
    g = (rng.standard_normal(n) * scale).astype(np.float32)
    g[rng.random(n) < 0.1] = 0.0
    m = (0.3 * rng.standard_normal(n) * scale).astype(np.float32)
    v = ((rng.standard_normal(n) * scale) ** 2).astype(np.float32)
    return rng.standard_normal(n).astype(np.float32), g, m, v


def formula(w, g, m, v, decay, c=1.0, alpha=1e-2, beta1=0.9, beta2=0.99, eps=1e-8, t=3):
    """(w, m, v, bars of the three) in fp64."""
    w, g, m, v = (np.asarray(x, dtype=np.float64) for x in (w, g, m, v))
    g = c * g
    bar_m = 5 * U * (beta1 * np.abs(m) + (1 - beta1) * np.abs(g)) + 2.0 ** -148
    bar_v = 7 * U * (beta2 * v + (1 - beta2) * g * g) + 2.0 ** -147
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    step = alpha / (1 - beta1 ** t)
    denom = np.sqrt(v) / np.sqrt(1 - beta2 ** t) + eps
    bar_w = 4 * U * np.abs(w) + step * (bar_m / denom + 16 * U * np.abs(m) / denom) + 2.0 ** -148
    return w * (1 - alpha * decay) - step * m / denom, m, v, bar_w, bar_m, bar_v


def near(got, want, bar):
    got = got.cpu().double().numpy()
    worst = np.max(np.abs(got - want) / bar) if got.size else 0.0
    assert worst <= 1.0, worst


@pytest.mark.parametrize("grad", TYPES)
@pytest.mark.parametrize("copy", [None, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("sizes", [[1], [3, 4, 5], [2047, 0, 2048, 2049], [100_003, 1, 64], [17] * 150])
def test_step(nuq, sizes, grad, copy):
    rng = np.random.default_rng(sum(sizes) + len(sizes))
    for shift, clip in ((0, False), (1, True), (3, False)):
        ws, gs, ms, vs, cs, want, decays = [], [], [], [], [], [], []
        c = np.float32(0.37) if clip else np.float32(1.0)
        for i, n in enumerate(sizes):
            w, g, m, v = vectors(n, rng)
            decays.append([0.1, 0.0, 0.5][i % 3])
            gs.append(to_dev(g, grad, shift))
            ws.append(to_dev(w, shift=shift))
            ms.append(to_dev(m, shift=shift + i % 2))
            vs.append(to_dev(v, shift=shift))
            cs.append(torch.full((n + 1,), 7.0, dtype=copy or torch.bfloat16, device=DEV)[1:])
            want.append(formula(w, gs[-1].float().cpu().numpy(), m, v, decays[-1], float(c), **HYPER))
        coefficient = torch.tensor([float(c)], device=DEV) if clip else None
        nuq.nuq_adamw_step(ws, gs, ms, vs, decays, *HYPER.values(), coefficient, cs if copy else None)
        for i in range(len(sizes)):
            w, m, v, bar_w, bar_m, bar_v = want[i]
            near(ws[i], w, bar_w)
            near(ms[i], m, bar_m)
            near(vs[i], v, bar_v)
            assert torch.equal(cs[i], ws[i].to(copy) if copy else torch.full_like(cs[i], 7.0))
    assert nuq.nuq_last_error_flags() == 0


def test_tensors_that_follow_each_other_and_the_same_apart(nuq):
    """Views into flat vectors (joined into runs where decay allows) against tensors of their own: the same bits."""
    rng = np.random.default_rng(5)
    sizes = [256, 512, 300, 1, 0, 4096, 255, 1024, 77]
    decays = [0.1, 0.1, 0.1, 0.0, 0.0, 0.0, 0.1, 0.1, 0.1]
    flat = [torch.from_numpy(x).to(DEV) for x in vectors(sum(sizes), rng)]
    split = lambda t: list(t.split(sizes))  # noqa: E731
    apart = [[x.clone() for x in split(t)] for t in flat]
    joined = [split(t) for t in flat]
    for ws, gs, ms, vs in (apart, joined):
        nuq.nuq_adamw_step(ws, gs, ms, vs, decays, *HYPER.values())
    for a, b in zip(apart, flat):
        assert torch.equal(torch.cat(a), b)


def test_several_steps_follow_the_formula(nuq):
    rng = np.random.default_rng(8)
    n = 3001
    w, _, _, _ = vectors(n, rng)
    m = v = np.zeros(n)
    tw, tm, tv = to_dev(w), torch.zeros(n, device=DEV), torch.zeros(n, device=DEV)
    w = w.astype(np.float64)
    for t in range(1, 21):
        g = rng.standard_normal(n).astype(np.float32)
        nuq.nuq_adamw_step([tw], [to_dev(g)], [tm], [tv], [0.01], 1e-2, 0.9, 0.999, 1e-8, t)
        w, m, v, *_ = formula(w, g, m, v, 0.01, alpha=1e-2, beta1=0.9, beta2=0.999, t=t)
    # every step adds its own bar; errors of earlier m and v fade with their betas
    near(tm, m, 20 * 5 * U * np.full(n, np.abs(m).max()))
    near(tv, v, 20 * 7 * U * np.full(n, v.max()))
    near(tw, w, 20 * (4 * U * np.abs(w).max() + 0.1 * 60 * U) * np.ones(n))


def test_what_is_not_finite_is_left_alone(nuq):
    n = 1000
    rng = np.random.default_rng(4)
    w, g, m, v = vectors(n, rng)
    g[[3, 500, 999]] = [np.inf, np.nan, 3e38]               # 3e38 squared is no float
    t = [to_dev(x) for x in (w, g, m, v)]
    copy = torch.zeros(n, dtype=torch.bfloat16, device=DEV)
    nuq.nuq_adamw_step(*([x] for x in t), None, *HYPER.values(), None, [copy])
    assert nuq.nuq_last_error_flags() == nuq.FLAG_NONFINITE
    bad = np.isin(np.arange(n), [3, 500, 999])
    for got, old in ((t[0], w), (t[2], m), (t[3], v)):
        assert np.array_equal(got.cpu().numpy()[bad], old[bad])
    assert torch.equal(copy, t[0].to(torch.bfloat16))
    want = formula(w[~bad], g[~bad], m[~bad], v[~bad], 0.0, **HYPER)
    near(t[0][torch.from_numpy(~bad).to(DEV)], want[0], want[3])
    # a factor that is NaN: nothing moves
    before = [x.clone() for x in t]
    nuq.nuq_adamw_step(*([x] for x in t), None, *HYPER.values(), torch.tensor([float("nan")], device=DEV))
    assert nuq.nuq_last_error_flags() == nuq.FLAG_NONFINITE
    assert all(torch.equal(a.nan_to_num(0.0), b.nan_to_num(0.0)) for a, b in zip(t, before))


# ---------------------------------------------------------------------------------------- states in 8 bits

def values_m():
    """e4m3 without sign: codes 0..126."""
    c = np.arange(127)
    e, f = c >> 3, c & 7
    return np.where(e > 0, (8 + f) * 2.0 ** (e - 10), f * 2.0 ** -9)


def values_v():
    c = np.arange(256)
    e, f = c >> 3, c & 7
    return np.where(e > 0, (8 + f) * 2.0 ** (e - 34), f * 2.0 ** -33)


def nearest(x, table):
    """Index of the entry nearest to x >= 0, ties to the even index."""
    hi = np.clip(np.searchsorted(table, x), 1, table.size - 1)
    lo = hi - 1
    a, b = x - table[lo], table[hi] - x
    return np.where((a < b) | ((a == b) & (lo % 2 == 0)), lo, hi)


def blocks_of(x):
    out = np.zeros((-(-x.size // 256), 256), dtype=np.float32)
    out.reshape(-1)[:x.size] = x
    return out


def held(codes_m, codes_v, scales):
    """fp32 values of codes."""
    n = codes_m.size
    a = scales.reshape(-1, 2)
    sign = np.where(codes_m & 0x80, np.float32(-1), np.float32(1))
    m = blocks_of(sign * values_m().astype(np.float32)[codes_m & 0x7F]) * (a[:, :1] * np.float32(2.0 ** -8))
    v = blocks_of(values_v().astype(np.float32)[codes_v]) * a[:, 1:]
    return m.reshape(-1)[:n], v.reshape(-1)[:n]


def to_codes(m, v):
    n = m.size
    m, v = blocks_of(m), blocks_of(v)
    a = np.stack([np.abs(m).max(1), v.max(1)], 1)
    a[a < 2.0 ** -126] = 0.0
    with np.errstate(divide="ignore"):
        inv = np.where(a > 0, np.float32(1.0) / a, np.float32(0.0)).astype(np.float32)
    y = m * inv[:, :1] * np.float32(256)
    cm = nearest(np.abs(y).astype(np.float64), values_m()) | np.where(np.signbit(y), 0x80, 0)
    z = (v * inv[:, 1:] * np.float32(2.0 ** -96)).astype(np.float64) * 2.0 ** 96
    cv = np.maximum(nearest(z, values_v()), (v > 0) & (a[:, 1:] > 0))
    return cm.reshape(-1)[:n].astype(np.uint8), cv.reshape(-1)[:n].astype(np.uint8), a.reshape(-1).astype(np.float32)


def moments32(g, m, v, c, beta1=0.9, beta2=0.99):
    f = np.float32
    g = g * f(c)
    return m * f(beta1) + g * f(1 - beta1), v * f(beta2) + g * g * f(1 - beta2)


def coded_state(m, v, shift=0):
    cm, cv, a = to_codes(m, v)
    tm = to_dev(cm, torch.uint8, shift).view(torch.float8_e4m3fn)
    return tm, to_dev(cv, torch.uint8, shift + shift), to_dev(a, shift=shift), held(cm, cv, a)


def check_coded(tm, tv, ta, m, v):
    cm, cv, a = to_codes(m, v)
    np.testing.assert_array_equal(ta.cpu().numpy(), a)
    np.testing.assert_array_equal(tv.cpu().numpy(), cv)
    np.testing.assert_array_equal(tm.view(torch.uint8).cpu().numpy(), cm)


@pytest.mark.parametrize("grad", TYPES)
@pytest.mark.parametrize("copy", [None, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("sizes", [[1], [2, 255, 256, 257], [1023, 0, 1024, 1025, 4095], [100_003, 4097], [300] * 130])
def test_coded_step(nuq, sizes, grad, copy):
    rng = np.random.default_rng(sum(sizes) + len(sizes))
    for shift, c in ((0, 1.0), (1, 0.37)):
        ws, gs, ms, vs, scales, cs, want, decays = [], [], [], [], [], [], [], []
        for i, n in enumerate(sizes):
            w, g, m, v = vectors(n, rng)
            decays.append([0.1, 0.0][i % 2])
            tm, tv, ta, (m, v) = coded_state(m, v, shift)
            ms.append(tm)
            vs.append(tv)
            scales.append(ta)
            ws.append(to_dev(w, shift=shift))
            gs.append(to_dev(g, grad, shift))
            cs.append(torch.zeros(n, dtype=copy or torch.bfloat16, device=DEV))
            g = gs[-1].float().cpu().numpy()
            want.append((formula(w, g, m, v, decays[-1], float(np.float32(c)), **HYPER), moments32(g, m, v, c)))
        coefficient = None if c == 1.0 else torch.tensor([c], device=DEV)
        nuq.nuq_adamw_step_coded(ws, gs, ms, vs, scales, decays, *HYPER.values(), coefficient, cs if copy else None)
        for i, n in enumerate(sizes):
            check_coded(ms[i], vs[i], scales[i], *want[i][1])
            near(ws[i], want[i][0][0], want[i][0][3])
            if copy:
                assert torch.equal(cs[i], ws[i].to(copy))
            m, v = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
            nuq.nuq_adamw_state_values(ms[i], vs[i], scales[i], m, v)
            mine = held(ms[i].view(torch.uint8).cpu().numpy(), vs[i].cpu().numpy(), scales[i].cpu().numpy())
            assert np.array_equal(m.cpu().numpy(), mine[0]) and np.array_equal(v.cpu().numpy(), mine[1])
    assert nuq.nuq_last_error_flags() == 0


def test_every_code_and_the_places_between(nuq):
    """Moments on every code, on every point halfway between two, and next to those; each block holds its scale's element."""
    points = []
    for table in (values_m() / 256, values_v()):
        table = table[table <= 1.0]
        mid = (table[1:] + table[:-1]) / 2
        x = np.concatenate([table, mid, np.nextafter(mid.astype(np.float32), np.float32(2)), np.nextafter(mid.astype(np.float32), np.float32(0))])
        points.append(np.resize(x.astype(np.float32), 1020))
    m = np.insert(points[0] * np.float32(0.25), [0, 255, 510, 765], 0.25).astype(np.float32)
    v = np.insert(points[1] * np.float32(0.0625), [0, 255, 510, 765], 0.0625).astype(np.float32)
    m[1::2] *= -1
    # gradients that put the moments there from a zero state: beta = 0, so m = g and v = g^2 are set one at a time
    n = m.size
    for beta1, g, tell in ((0.0, m, "m"), (0.5, np.sqrt(v.astype(np.float64)).astype(np.float32), "v")):
        tm = torch.zeros(n, dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn)
        tv, ta = torch.zeros(n, dtype=torch.uint8, device=DEV), torch.zeros(2 * 4 + 2 * (n > 1024), device=DEV)
        nuq.nuq_adamw_step_coded([torch.zeros(n, device=DEV)], [to_dev(g)], [tm], [tv], [ta], None, 1e-3, beta1, 0.0, 1e-8, 1)
        check_coded(tm, tv, ta, *moments32(g, np.zeros(n, np.float32), np.zeros(n, np.float32), 1.0, beta1, 0.0))
        if tell == "m":
            assert len(np.unique(tm.view(torch.uint8).cpu().numpy() & 0x7F)) == 121     # all up to the scale's own, 0x78
    assert nuq.nuq_last_error_flags() == 0


def test_extreme_blocks(nuq):
    """Blocks of zeros, of a single element, too small to scale, at the edge of that, and of huge values; a tiny v above zero
    beside a huge one stays above zero."""
    g = np.zeros((7, 256), dtype=np.float32)
    g[1, 17] = -3.0
    g[2] = 1e-30                       # v = 1e-62: nothing; m below 2^-126 only in parts
    g[3] = 2e-38
    g[4] = np.linspace(-1e18, 1e18, 256)
    g[5] = 1e-7
    g[5, 0] = 1e3
    g[6, :128] = 1.5e-19               # v around the smallest normal float
    g[6, 128:] = 9e-19
    g = g.reshape(-1)[:-3]
    n = g.size
    tm = torch.zeros(n, dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn)
    tv, ta, w = torch.zeros(n, dtype=torch.uint8, device=DEV), torch.zeros(14, device=DEV), torch.ones(n, device=DEV)
    m = v = np.zeros(n, dtype=np.float32)
    for t in range(1, 4):
        before = w.cpu().numpy()
        nuq.nuq_adamw_step_coded([w], [to_dev(g)], [tm], [tv], [ta], [0.0], 1e-3, 0.9, 0.99, 1e-8, t)
        m, v = moments32(g, m, v, 1.0)
        check_coded(tm, tv, ta, m, v)
        want = formula(before, g, *held(*[np.zeros(n, np.uint8)] * 2, np.zeros(14, np.float32)), 0.0, t=t, alpha=1e-3) if t == 1 else None
        if want:
            near(w, want[0], want[3])
        m, v = held(tm.view(torch.uint8).cpu().numpy(), tv.cpu().numpy(), ta.cpu().numpy())
        assert np.all(v.reshape(-1)[5 * 256:6 * 256] > 0)
        assert np.all(np.abs(w.cpu().numpy() - before) <= 1.5e-3)          # no step is much longer than alpha
    assert nuq.nuq_last_error_flags() == 0


def test_a_block_that_is_not_finite_is_left_alone(nuq):
    rng = np.random.default_rng(6)
    n = 256 * 9 + 40
    w, g, m, v = vectors(n, rng)
    g[256 * 2 + 5], g[256 * 9 + 39], g[256 * 4] = np.nan, -np.inf, 1e30
    tm, tv, ta, (m, v) = coded_state(m, v)
    tw, copy = to_dev(w), torch.zeros(n, dtype=torch.float16, device=DEV)
    old = [x.clone() for x in (tw, tm.view(torch.uint8), tv, ta)]
    nuq.nuq_adamw_step_coded([tw], [to_dev(g)], [tm], [tv], [ta], None, *HYPER.values(), None, [copy])
    assert nuq.nuq_last_error_flags() == nuq.FLAG_NONFINITE
    at = np.isin(np.arange(n) // 256, [2, 4, 9])
    mask = torch.from_numpy(at).to(DEV)
    for got, was in zip((tw, tm.view(torch.uint8), tv), old):
        assert torch.equal(got[mask], was[mask]) and not torch.equal(got[~mask], was[~mask])
    assert torch.equal(ta.view(-1, 2)[[2, 4, 9]], old[3].view(-1, 2)[[2, 4, 9]])
    assert torch.equal(copy, tw.half())
    want = formula(w[~at], g[~at], m[~at], v[~at], 0.0, **HYPER)
    near(tw[~mask], want[0], want[3])


def test_coded_training_comes_as_low_as_uncoded(nuq):
    """A noisy quadratic from a distance of 1: both come within a tenth of it."""
    n, far = 4096, {}
    for coded in (False, True):
        g = torch.Generator(device=DEV).manual_seed(1)
        w = torch.zeros(n, device=DEV)
        target = torch.randn(n, generator=g, device=DEV)
        curve = 10.0 ** torch.empty(n, device=DEV).uniform_(-1, 1, generator=g)
        m = torch.zeros(n, dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn) if coded else torch.zeros(n, device=DEV)
        v = torch.zeros(n, dtype=torch.uint8, device=DEV) if coded else torch.zeros(n, device=DEV)
        scales = torch.zeros(2 * n // 256, device=DEV)
        for t in range(1, 801):
            grad = curve * (w - target + 0.1 * torch.randn(n, generator=g, device=DEV))
            alpha = 2e-2 * (1.0 - t / 801)
            if coded:
                nuq.nuq_adamw_step_coded([w], [grad], [m], [v], [scales], None, alpha, 0.9, 0.95, 1e-8, t)
            else:
                nuq.nuq_adamw_step([w], [grad], [m], [v], None, alpha, 0.9, 0.95, 1e-8, t)
        far[coded] = float((w - target).square().mean().sqrt())
    assert max(far.values()) < 0.1, far


# ---------------------------------------------------------------------------------------- the norm

@pytest.mark.parametrize("grad", TYPES)
@pytest.mark.parametrize("sizes", [[], [0], [1], [3, 0, 5], [4095, 4096, 4097], [1_000_003, 17], [11] * 300])
def test_gradient_norm(nuq, sizes, grad):
    rng = np.random.default_rng(len(sizes) + sum(sizes))
    ws, out = torch.empty(nuq.GRADIENT_NORM_WORKSPACE_BYTES, dtype=torch.uint8, device=DEV), torch.empty(2, device=DEV)
    gs = [to_dev((rng.standard_normal(n) * 3).astype(np.float32), grad, i % 3) for i, n in enumerate(sizes)]
    want = np.sqrt(sum(float(x.double().square().sum()) for x in gs))
    for limit in (1.0, 1e9, float("inf")):
        nuq.nuq_gradient_norm(gs, limit, ws, out)
        norm, c = out.tolist()
        assert abs(norm - want) <= 2 * U * want
        assert c == (1.0 if want <= limit else pytest.approx(limit / want, rel=2 * U))
    first = out.clone()
    for _ in range(3):
        nuq.nuq_gradient_norm(gs, float("inf"), ws, out)
        assert torch.equal(out, first)                       # a fixed order: the same bits
    assert nuq.nuq_last_error_flags() == 0


def test_gradient_norm_of_large_and_of_no_finite_values(nuq):
    ws, out = torch.empty(nuq.GRADIENT_NORM_WORKSPACE_BYTES, dtype=torch.uint8, device=DEV), torch.empty(2, device=DEV)
    nuq.nuq_gradient_norm([torch.full((1000,), 1e30, device=DEV), torch.full((8,), 1e-42, device=DEV)], 1.0, ws, out)
    assert out.tolist() == [pytest.approx(1e30 * 1000 ** 0.5, rel=2 * U), pytest.approx(1e-30 / 1000 ** 0.5, rel=2 * U)]
    assert nuq.nuq_last_error_flags() == 0
    for bad in (float("inf"), float("nan"), 3e38):           # two of the last: the norm is no float
        nuq.nuq_gradient_norm([torch.ones(5, device=DEV), torch.full((2,), bad, device=DEV)], 1.0, ws, out)
        norm, c = out.tolist()
        assert not np.isfinite(norm) and np.isnan(c)
        assert nuq.nuq_last_error_flags() == nuq.FLAG_NONFINITE


def test_offsets_beyond_32_bits(nuq):
    """More than 2^32 bytes of weights and 2^31 bytes of gradients: the tail of a long tensor moves as a short one does."""
    n, tail = (1 << 30) + 5 * 256 + 3, 256 * 7 + 3
    gen = torch.Generator(device=DEV).manual_seed(2)
    w = torch.zeros(n, device=DEV)
    g = torch.zeros(n, dtype=torch.bfloat16, device=DEV)
    w[-tail:].normal_(generator=gen)
    g[-tail:] = torch.randn(tail, generator=gen, device=DEV).bfloat16()
    g[0] = 1.0
    m, v = torch.zeros(n, dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn), torch.zeros(n, dtype=torch.uint8, device=DEV)
    scales = torch.zeros(2 * nuq.nuq_state_blocks(n), device=DEV)
    short = [x[-tail:].clone() for x in (w, g)]
    small = torch.zeros(tail, dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn), torch.zeros(tail, dtype=torch.uint8, device=DEV)
    few = torch.zeros(2 * nuq.nuq_state_blocks(tail), device=DEV)
    nuq.nuq_adamw_step_coded([w], [g], [m], [v], [scales], [0.1], *HYPER.values())
    nuq.nuq_adamw_step_coded([short[0]], [short[1]], [small[0]], [small[1]], [few], [0.1], *HYPER.values())
    assert torch.equal(w[-tail:], short[0]) and torch.equal(v[-tail:], small[1]) and torch.equal(scales[-few.numel():], few)
    assert torch.equal(m.view(torch.uint8)[-tail:], small[0].view(torch.uint8))
    assert w[0].item() < 0 and not w[1:1000].any()
    ws, out = torch.empty(nuq.GRADIENT_NORM_WORKSPACE_BYTES, dtype=torch.uint8, device=DEV), torch.empty(2, device=DEV)
    nuq.nuq_gradient_norm([g], 1.0, ws, out)
    assert out[0].item() == pytest.approx((1.0 + float(short[1].double().square().sum())) ** 0.5, rel=2 * U)
    del m, v, scales
    m, v = torch.zeros(n, device=DEV), torch.zeros(n, device=DEV)
    w[-tail:].normal_(generator=gen)
    short[0] = w[-tail:].clone()
    some = torch.zeros(tail, device=DEV), torch.zeros(tail, device=DEV)
    nuq.nuq_adamw_step([w], [g], [m], [v], [0.1], *HYPER.values())
    nuq.nuq_adamw_step([short[0]], [short[1]], [some[0]], [some[1]], [0.1], *HYPER.values())
    assert torch.equal(w[-tail:], short[0]) and torch.equal(m[-tail:], some[0]) and torch.equal(v[-tail:], some[1])


def test_steps_on_a_stream_of_their_own_and_in_a_graph(nuq):
    """The calls run on the current stream; captured, they replay as the eager calls go."""
    rng = np.random.default_rng(9)
    n = 50_001
    w, g, m, v = vectors(n, rng)
    out, ws = torch.empty(2, device=DEV), torch.empty(nuq.GRADIENT_NORM_WORKSPACE_BYTES, dtype=torch.uint8, device=DEV)

    def step(t):
        nuq.nuq_gradient_norm([t[1]], 1.0, ws, out)
        nuq.nuq_adamw_step([t[0]], [t[1]], [t[2]], [t[3]], None, *HYPER.values(), out[1:])
    eager, replayed = ([to_dev(x) for x in (w, g, m, v)] for _ in range(2))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(replayed)                                       # (on a stream of its own, uncaptured)
    torch.cuda.current_stream().wait_stream(side)
    step(eager)
    assert all(torch.equal(a, b) for a, b in zip(eager, replayed))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(replayed)
    for k in range(4):
        new = torch.from_numpy(vectors(n, rng)[1]).to(DEV)
        for t in (eager, replayed):
            t[1].copy_(new)
        graph.replay()
        step(eager)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, replayed))
