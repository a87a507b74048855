"""Softmax cross entropy of a large vocabulary against its formula in 64 bits, forward and backward.

Bars.  u = 2^-24.  A logit is a sum of H products, each exact (16 bits) or rounded to u (fp32), added in fp32 one after the other:
H u of the summed magnitudes |x| |w| at most, 2 H u for fp32 operands (the matrix cores may cut instead of round: a unit, not half a unit,
so twice that).  lse moves by no more than the largest error of a row's logits; exponentials and their sums add 16 u and 256 u of 1
(relative to the sum, so absolute in lse), the maximum's and the result's rounding 4 u of their magnitude.
d: exp(z - lse) is off by the factor 1 + (error of z) + 4 u (1 + |z - lse|), then d is rounded to the type (half a unit, of d less what
is subtracted), in fp16 to 2^-24 / 2^14 at least.  dx, dw: these errors through the products, (terms + 2) u of the summed magnitudes, twice, and
half a unit of the result; the factor g over the largest |g| adds u, and a half unit of the type for the product with it."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")
U = 2.0 ** -24
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
HALF_UNIT = {F32: 2.0 ** -24, BF16: 2.0 ** -8, F16: 2.0 ** -11}
LEAST = {F32: 2.0 ** -140, BF16: 2.0 ** -126, F16: 2.0 ** -24}
LEAST_D = {F32: 2.0 ** -140, BF16: 2.0 ** -126, F16: 2.0 ** -38}
# rows, hidden, vocabulary
SHAPES = [(1, 1, 1), (1, 8, 2), (3, 7, 5), (1, 64, 1000), (2, 1600, 50257), (17, 129, 257), (32, 64, 256), (33, 72, 300), (64, 128, 4097),
          (65, 65, 513), (128, 100, 129), (129, 64, 1023), (200, 200, 2000), (257, 1001, 777), (300, 40, 10007), (513, 320, 1500)]


@pytest.fixture(scope="module")
def nuq():
    import paper_1908_06077_amd
    return paper_1908_06077_amd


def close(got, want, bar, what=""):
    if got.numel():
        off = (got.double() - want).abs()
        worst = float((off / bar).max())
        assert worst <= 1.0, (what, worst)


def inputs(rows, hidden, vocab, kind, seed, pad=0, ignored=True):
    g = torch.Generator(device=DEV).manual_seed(seed)
    w = torch.randn(vocab, hidden + pad, generator=g, device=DEV) * (2.0 / hidden ** 0.5)
    target = torch.randint(0, vocab, (rows,), generator=g, device=DEV)
    x = (torch.randn(rows, hidden + pad, generator=g, device=DEV) + 1.2 * w[target]).to(kind)
    if ignored and rows > 2:
        target[1::5] = -100
    return x[:, pad // 2:pad // 2 + hidden], w.to(kind)[:, pad // 2:pad // 2 + hidden], target


def formula(x, w, target, smoothing):
    """(z, lse, loss, bar of z, of lse, of loss) in fp64."""
    kind, (rows, hidden), vocab = x.dtype, x.shape, w.shape[0]
    x, w = x.double(), w.double()
    z = x @ w.t()
    bar = (2 if kind != F32 else 4) * (hidden + 2) * U * (x.abs() @ w.abs().t()) + 2.0 ** -140
    lse = torch.logsumexp(z, 1)
    bar_lse = bar.amax(1) + 272 * U + 4 * U * (lse.abs() + z.abs().amax(1))
    valid = target != -100
    at = target.clamp(min=0)[:, None]
    loss = (1 - smoothing) * (lse - z.gather(1, at)[:, 0]) + smoothing * (lse - z.mean(1))
    bar_loss = bar_lse + bar.amax(1) + 8 * U * (lse.abs() + z.abs().amax(1)) + (256 + vocab / 64) * U * smoothing * z.abs().mean(1)
    return z, lse, torch.where(valid, loss, torch.zeros_like(loss)), bar, bar_lse, bar_loss


def forward(nuq, x, w, target, smoothing=0.0, ignore=-100, mean=True):
    rows = x.shape[0]
    ws = torch.full((nuq.nuq_linear_cross_entropy_workspace_bytes(x, w, False),), 255, dtype=torch.uint8, device=DEV)
    loss, lse, m = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV), torch.empty(2, device=DEV) if mean else None
    nuq.nuq_linear_cross_entropy_forward(x, w, target, ignore, smoothing, loss, lse, m, ws)
    return loss, lse, m


def backward(nuq, x, w, target, lse, grad, mean=None, smoothing=0.0, ignore=-100, dx=True, dw=True):
    ws = torch.full((nuq.nuq_linear_cross_entropy_workspace_bytes(x, w, True),), 255, dtype=torch.uint8, device=DEV)
    a = torch.full((x.shape[0], x.shape[1] + 3), 7.0, dtype=x.dtype, device=DEV) if dx else None
    b = torch.full((w.shape[0], w.shape[1] + 3), 7.0, dtype=x.dtype, device=DEV) if dw else None
    cut = lambda t: None if t is None else t[:, :x.shape[1]]  # noqa: E731
    nuq.nuq_linear_cross_entropy_backward(x, w, target, ignore, smoothing, lse, grad, mean, cut(a), cut(b), ws)
    for t in (a, b):
        assert t is None or (t[:, x.shape[1]:] == 7.0).all()
    return cut(a), cut(b)


@pytest.mark.parametrize("kind", [F32, BF16, F16])
@pytest.mark.parametrize("rows,hidden,vocab", SHAPES)
def test_forward(nuq, rows, hidden, vocab, kind):
    for pad, smoothing in ((0, 0.0), (3, 0.1), (8, 0.0)):
        x, w, target = inputs(rows, hidden, vocab, kind, rows + hidden, pad)
        loss, lse, mean = forward(nuq, x, w, target, smoothing)
        _, want_lse, want, _, bar_lse, bar = formula(x, w, target, smoothing)
        close(lse, want_lse, bar_lse, "lse")
        close(loss, want, bar, "loss")
        valid = target != -100
        assert not loss[~valid].any()
        count = int(valid.sum())
        assert abs(float(mean[0]) - float(loss.double().sum()) / count) <= 4 * U * float(loss.double().abs().sum()) / count
        assert float(mean[1]) == float(torch.tensor(1.0 / count, dtype=F32))
    assert nuq.nuq_last_error_flags() == 0


def gradient_formula(x, w, target, lse, g, smoothing, per_row=False):
    """((dx, bar), (dw, bar)) in fp64."""
    kind, (rows, hidden), vocab = x.dtype, x.shape, w.shape[0]
    z, _, _, bar_z, _, _ = formula(x, w, target, smoothing)
    x, w, lse = x.double(), w.double(), lse.double()[:, None]
    p = (z - lse).exp()
    d = p - smoothing / vocab
    d.scatter_add_(1, target.clamp(min=0)[:, None], torch.full_like(lse, smoothing - 1.0))
    wanted = torch.full_like(p, smoothing / vocab)
    wanted.scatter_add_(1, target.clamp(min=0)[:, None], torch.full_like(lse, 1.0 - smoothing))
    bar = p * (bar_z * 1.01 + 4 * U * (2 + (z - lse).abs() + lse.abs())) + 4 * U * wanted + LEAST_D[kind]
    bar = bar + HALF_UNIT[kind] * (1 + 4 * U) * (d.abs() + bar)
    valid = (target != -100)[:, None]
    g = torch.where(valid[:, 0], g.double().expand(rows), torch.zeros_like(lse[:, 0]))[:, None]
    d, bar = d * valid, bar * valid
    dx = d @ w * g
    bar_x = (bar @ w.abs() + 2 * (vocab + 66) * U * (d.abs() @ w.abs())) * g.abs() + 6 * U * dx.abs()
    gd, top = g * d, float(g.abs().max())
    bar_d = g.abs() * bar + 4 * U * gd.abs() + ((HALF_UNIT[kind] * (g.abs() * bar + gd.abs()) + top * LEAST_D[kind]) if per_row else 0.0)
    dw = gd.t() @ x
    bar_w = bar_d.t() @ x.abs() + 2 * (rows + 2) * U * (gd.abs().t() @ x.abs()) + 4 * U * dw.abs()
    half = lambda v, b: b + HALF_UNIT[kind] * (1 + 4 * U) * (v.abs() + b) + LEAST[kind]  # noqa: E731
    return (dx, half(dx, bar_x)), (dw, half(dw, bar_w))


@pytest.mark.parametrize("kind", [F32, BF16, F16])
@pytest.mark.parametrize("rows,hidden,vocab", SHAPES)
def test_backward(nuq, rows, hidden, vocab, kind):
    for pad, smoothing, per_row in ((0, 0.0, False), (3, 0.1, True), (8, 0.0, False)):
        x, w, target = inputs(rows, hidden, vocab, kind, rows + hidden, pad)
        lse = formula(x, w, target, smoothing)[1].float()
        gen = torch.Generator(device=DEV).manual_seed(3)
        mean = torch.tensor([0.0, 1.0 / max(1, int((target != -100).sum()))], device=DEV)
        grad = torch.randn(rows, generator=gen, device=DEV) if per_row and rows > 1 else torch.tensor([0.7], device=DEV)
        dx, dw = backward(nuq, x, w, target, lse, grad, mean, smoothing)
        (want_x, bar_x), (want_w, bar_w) = gradient_formula(x, w, target, lse, grad.double() * mean[1].double(), smoothing, per_row and rows > 1)
        close(dx, want_x, bar_x, "dx")
        close(dw, want_w, bar_w, "dw")
        alone = backward(nuq, x, w, target, lse, grad, mean, smoothing, dw=False)[0]
        assert torch.equal(alone, dx)
        alone = backward(nuq, x, w, target, lse, grad, mean, smoothing, dx=False)[1]
        assert torch.equal(alone, dw)
    assert nuq.nuq_last_error_flags() == 0


@pytest.mark.parametrize("kind", [BF16, F32])
def test_several_pieces_of_the_vocabulary(nuq, kind):
    """More rows than one piece of the whole vocabulary leaves room for."""
    rows, hidden, vocab = 4100, 96, 20011
    x, w, target = inputs(rows, hidden, vocab, kind, 5)
    loss, lse, mean = forward(nuq, x, w, target)
    _, want_lse, want, _, bar_lse, bar = formula(x, w, target, 0.0)
    close(lse, want_lse, bar_lse, "lse")
    close(loss, want, bar, "loss")
    one = torch.ones(1, device=DEV)
    dx, dw = backward(nuq, x, w, target, lse, one, mean)
    (want_x, bar_x), (want_w, bar_w) = gradient_formula(x, w, target, lse, mean[1], 0.0)
    close(dx, want_x, bar_x, "dx")
    close(dw, want_w, bar_w, "dw")
    again = backward(nuq, x, w, target, lse, one, mean)
    assert torch.equal(again[0], dx) and torch.equal(again[1], dw)           # a fixed order: the same bits


def test_gradients_far_apart_in_fp16(nuq):
    """Rows whose gradients differ by 2^20 beside a large vocabulary: a small row's own gradient keeps its digits."""
    rows, hidden, vocab = 40, 64, 30000
    x, w, target = inputs(rows, hidden, vocab, F16, 6, ignored=False)
    lse = forward(nuq, x, w, target)[1]
    grad = torch.ones(rows, device=DEV)
    grad[::2] = 2.0 ** -8
    dx, dw = backward(nuq, x, w, target, lse, grad)
    (want_x, bar_x), (want_w, bar_w) = gradient_formula(x, w, target, lse, grad, 0.0, True)
    close(dx, want_x, bar_x, "dx")
    close(dw, want_w, bar_w, "dw")


def test_rows_that_do_not_count(nuq):
    rows, hidden, vocab = 70, 128, 999
    for kind in (BF16, F32):
        x, w, target = inputs(rows, hidden, vocab, kind, 7)
        x = x.clone()
        clean = forward(nuq, x, w, target)
        one = torch.ones(1, device=DEV)
        grads = backward(nuq, x, w, target, clean[1], one, clean[2])
        x[1, 5], x[6, 0], x[11] = float("nan"), float("inf"), -float("inf")        # rows that are ignored
        got = forward(nuq, x, w, target)
        valid = target != -100
        assert torch.equal(got[0], clean[0]) and torch.equal(got[1][valid], clean[1][valid]) and torch.equal(got[2], clean[2])
        again = backward(nuq, x, w, target, got[1], one, got[2])
        assert torch.equal(again[0], grads[0]) and torch.equal(again[1], grads[1]) and not again[0][~valid].any()
        # none counts
        none = torch.full_like(target, -100)
        loss, lse, mean = forward(nuq, x, w, none)
        assert not loss.any() and mean.tolist() == [0.0, 1.0]
        again = backward(nuq, x, w, none, lse, one, mean)
        assert not again[0].any() and not again[1].any()
        assert nuq.nuq_last_error_flags() == 0
        # a target outside the vocabulary
        for bad in (vocab, -1, 2 ** 40, -2 ** 62):
            wrong = target.clone()
            wrong[2] = bad
            loss, lse, mean = forward(nuq, x, w, wrong)
            assert nuq.nuq_last_error_flags() == nuq.FLAG_MALFORMED
            assert loss[2].isnan() and mean[0].isnan() and torch.equal(loss[[0, 3, 4]], clean[0][[0, 3, 4]])
            dx, _ = backward(nuq, x, w, wrong, lse, one, mean)
            assert nuq.nuq_last_error_flags() == nuq.FLAG_MALFORMED
            assert not dx[2].any() and torch.equal(dx[[0, 3, 4]], grads[0][[0, 3, 4]])
        # another number stands for what is ignored, also one inside the vocabulary
        for ignore in (0, 5, -1):
            other = torch.where(target == -100, torch.full_like(target, ignore), target)
            valid = other != ignore
            loss, _, mean = forward(nuq, x, w, other, ignore=ignore)
            assert torch.equal(loss[valid], clean[0][valid]) and not loss[~valid].any()


def test_extreme_logits(nuq):
    """Logits of +-1e4 and equal ones: no overflow, and the sum is over all of the vocabulary."""
    w = torch.zeros(700, 8, device=DEV)
    w[5, 0], w[600, 0] = 1e4, -1e4
    x = torch.zeros(4, 8, device=DEV)
    x[0, 0], x[1, 0] = 1.0, -1.0
    target = torch.tensor([5, 5, 7, 699], device=DEV)
    loss, lse, _ = forward(nuq, x, w, target)
    want = torch.tensor([0.0, 2e4, 700.0, 700.0], dtype=torch.float64, device=DEV)
    want[2:] = want[2:].log()
    assert float((loss.double() - want).abs().max()) <= 64 * U * 7 and torch.equal(lse[:2], torch.tensor([1e4, 1e4], device=DEV))
    x[2, 1], w[3, 1] = 1.0, float("inf")                     # an infinite logit: lse is infinite, its row alone
    w[4, 1] = -float("inf")
    x[:, 1] += 1.0
    x[[0, 1, 3], 1] = 0.0
    out = forward(nuq, x[2:3], w, target[2:3])
    assert float(out[1][0]) == float("inf") and float(out[0][0]) == float("inf")


@pytest.mark.parametrize("kind", [F32, BF16])
def test_rows_that_overlap(nuq, kind):
    """Strides of zero (one row for all), one element and sixteen bytes."""
    rows, hidden, vocab = 40, 64, 300
    x, w, target = inputs(rows, hidden, vocab, kind, 3, ignored=False)
    flat, many = torch.randn(4096, device=DEV).to(kind), torch.randn(8192, device=DEV).to(kind) / 4
    one = torch.ones(1, device=DEV)
    for stride in (0, 1, 8):
        xs, ws = flat.as_strided((rows, hidden), (stride, 1)), many.as_strided((vocab, hidden), (stride, 1))
        for a, b in ((xs, w), (x, ws), (xs, ws), (x[:1].expand(1, hidden), w)):
            t = target[:a.shape[0]]
            got, want = forward(nuq, a, b, t), forward(nuq, a.contiguous(), b.contiguous(), t)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
            g, h = backward(nuq, a, b, t, got[1], one, got[2]), backward(nuq, a.contiguous(), b.contiguous(), t, got[1], one, got[2])
            assert torch.equal(g[0], h[0]) and torch.equal(g[1], h[1])


def test_no_rows(nuq):
    x, w = torch.empty(0, 24, device=DEV), torch.randn(50, 24, device=DEV)
    target, mean = torch.empty(0, dtype=torch.int64, device=DEV), torch.empty(2, device=DEV)
    ws = torch.empty(16, dtype=torch.uint8, device=DEV)
    lse = torch.empty(0, device=DEV)
    nuq.nuq_linear_cross_entropy_forward(x, w, target, -100, 0.0, None, lse, mean, ws)
    assert mean.tolist() == [0.0, 1.0]
    dw = torch.full_like(w, 7.0)
    nuq.nuq_linear_cross_entropy_backward(x, w, target, -100, 0.0, lse, torch.ones(1, device=DEV), mean, torch.empty_like(x), dw, ws)
    assert not dw.any()


def test_offsets_beyond_32_bits(nuq):
    """Rows and weights at strides that put the last beyond 2^32 elements."""
    hidden, rows, vocab = 64, 3, 5
    x, w, target = inputs(rows, hidden, vocab, BF16, 9)
    for stride in ((1 << 31) + 16, (1 << 31) + 17):
        far = torch.zeros(stride * 2 + hidden, dtype=BF16, device=DEV).as_strided((rows, hidden), (stride, 1))
        far.copy_(x)
        a, b = forward(nuq, x, w, target), forward(nuq, far, w, target)
        assert torch.equal(a[0], b[0])
        one = torch.ones(1, device=DEV)
        g, h = backward(nuq, x, w, target, a[1], one, a[2]), backward(nuq, far, w, target, a[1], one, a[2])
        assert torch.equal(g[0], h[0]) and torch.equal(g[1], h[1])


# ---------------------------------------------------------------------------------------- the module

def test_module_gradients_against_differences(nuq):
    from paper_1908_06077_amd.loss import LinearCrossEntropy
    hidden, vocab, rows, h = 12, 50, 9, 1e-5
    gen = torch.Generator(device=DEV).manual_seed(2)
    x = torch.randn(3, 3, hidden, generator=gen, device=DEV, requires_grad=True)
    target = torch.randint(0, vocab, (3, 3), generator=gen, device=DEV)
    target[1, 1] = -100
    for reduction in ("mean", "none"):
        head = LinearCrossEntropy(hidden, vocab, smoothing=0.1, device=DEV)
        weights = torch.rand(3, 3, generator=gen, device=DEV, dtype=torch.float64)
        x.grad = None
        loss = head(x, target, reduction)
        assert loss.shape == (() if reduction == "mean" else target.shape)
        (loss if reduction == "mean" else (loss * weights.float()).sum()).backward()

        def value(x, w):
            z = x.reshape(rows, hidden) @ w.t()
            lse, t = torch.logsumexp(z, 1), target.view(-1)
            each = lse - 0.9 * z.gather(1, t.clamp(min=0)[:, None])[:, 0] - 0.1 * z.mean(1)
            each = each * (t != -100)
            return float(each.sum() / (t != -100).sum() if reduction == "mean" else (each * weights.view(-1)).sum())
        both = [x.detach().double(), head.weight.detach().double()]
        for k, grad in enumerate((x.grad, head.weight.grad)):
            for at in range(0, grad.numel(), 11):
                ends = []
                for sign in (1, -1):
                    moved = [t.clone() for t in both]
                    moved[k].view(-1)[at] += sign * h
                    ends.append(value(*moved))
                slope = (ends[0] - ends[1]) / (2 * h)
                assert abs(float(grad.reshape(-1)[at]) - slope) <= 1e-5 * (1.0 + abs(slope)), (k, at)


def test_module_types_and_refusals(nuq):
    from paper_1908_06077_amd.loss import LinearCrossEntropy, linear_cross_entropy
    head = LinearCrossEntropy(48, 300, device=DEV)
    gen = torch.Generator(device=DEV).manual_seed(2)
    x = torch.randn(48, 5, generator=gen, device=DEV, dtype=BF16).t().requires_grad_()       # rows that are not contiguous
    target = torch.randint(0, 300, (5,), generator=gen, device=DEV)
    loss = head(x, target)                                   # fp32 weights beside rows in bfloat16
    loss.backward()
    assert loss.dtype == F32 and x.grad.dtype == BF16 and head.weight.grad.dtype == F32 and head.weight.grad.isfinite().all()
    want = torch.nn.functional.cross_entropy(x.detach().cpu().double() @ head.weight.detach().to(BF16).cpu().double().t(), target.cpu())
    assert abs(float(loss.detach()) - float(want)) <= 1e-4
    one = linear_cross_entropy(x[:1], head.weight, target[:1], reduction="none")
    one.sum().backward()
    frozen = LinearCrossEntropy(48, 300, device=DEV).requires_grad_(False)
    x.grad = None
    frozen(x, target).backward()
    assert frozen.weight.grad is None and x.grad is not None
    for bad in (lambda: head(x, target[:4]), lambda: head(x[:, :47], target), lambda: head(x, target.int()),
                lambda: linear_cross_entropy(x, head.weight, target, reduction="sum"), lambda: LinearCrossEntropy(4, 4, smoothing=1.0)):
        with pytest.raises(ValueError):
            bad()


def test_forward_and_backward_replay_in_a_graph(nuq):
    rows, hidden, vocab = 300, 200, 5003
    x, w, target = inputs(rows, hidden, vocab, BF16, 1)
    loss, lse, mean = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV), torch.empty(2, device=DEV)
    one, dx, dw = torch.ones(1, device=DEV), torch.empty_like(x), torch.empty_like(w)
    ws = torch.empty(max(nuq.nuq_linear_cross_entropy_workspace_bytes(x, w, b) for b in (False, True)), dtype=torch.uint8, device=DEV)

    def both():
        nuq.nuq_linear_cross_entropy_forward(x, w, target, -100, 0.0, loss, lse, mean, ws)
        nuq.nuq_linear_cross_entropy_backward(x, w, target, -100, 0.0, lse, one, mean, dx, dw, ws)
    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for _ in range(4):
        x.normal_()
        both()
        out = (loss, lse, mean, dx, dw)
        want = [t.clone() for t in out]
        for t in out:
            t.zero_()
        ws.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, out))


def both_ways(nuq, rows, hidden, vocab, kind, smoothing=0.0, pad=0):
    x, w, target = inputs(rows, hidden, vocab, kind, rows + hidden + vocab, pad)
    loss, lse, mean = forward(nuq, x, w, target, smoothing)
    _, want_lse, want, _, bar_lse, bar = formula(x, w, target, smoothing)
    what = (rows, hidden, vocab)
    close(lse, want_lse, bar_lse, ("lse", *what))
    close(loss, want, bar, ("loss", *what))
    dx, dw = backward(nuq, x, w, target, lse, torch.ones(1, device=DEV), mean, smoothing)
    (want_x, bar_x), (want_w, bar_w) = gradient_formula(x, w, target, lse, mean[1], smoothing)
    close(dx, want_x, bar_x, ("dx", *what))
    close(dw, want_w, bar_w, ("dw", *what))


@pytest.mark.parametrize("kind", [F32, BF16, F16])
@pytest.mark.parametrize("rows", [5, 40, 70])
def test_every_number_of_steps(nuq, rows, kind):
    """Depths of one step, of as many as there are stages, of one less and one more, whole and cut: in the logits over the width, in the
    gradients over the vocabulary and the rows."""
    for hidden in (1, 33, 64, 65, 96, 128, 129, 192, 193, 257, 320, 385):
        both_ways(nuq, rows, hidden, 203, kind)
    for vocab in (1, 31, 64, 65, 96, 128, 129, 192, 257, 320, 385):
        both_ways(nuq, rows, 72, vocab, kind, 0.1)


@pytest.mark.parametrize("kind", [F32, BF16, F16])
@pytest.mark.parametrize("rows", [1, 31, 63, 65, 96, 127, 129, 192, 200, 257, 321])
def test_every_number_of_rows(nuq, rows, kind):
    both_ways(nuq, rows, 136, 140, kind)


@pytest.mark.parametrize("kind", [F32, BF16])
@pytest.mark.parametrize("rows,hidden,vocab", [(70, 1001, 8300), (2600, 40, 8300), (2600, 72, 8300), (2600, 136, 8300)])
def test_largest_tiles(nuq, rows, hidden, vocab, kind):
    """Enough tiles that the largest are taken, in the weights' gradient and in the logits, with depths of a step and of a few."""
    both_ways(nuq, rows, hidden, vocab, kind)
    both_ways(nuq, rows, hidden, vocab, kind, 0.1, pad=3)
