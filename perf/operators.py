"""The operators of transformer training as measurable cases: one case is one pass through one of them at one size.

Paths (one pass each):
  adamw        a parameter step: AdamW over many tensors, states in 32 bits; where `clip`, behind the norm of all gradients
  adamw_coded  the same with both states in 8 bits; the states come back as the values that their codes stand for
  norm         the norm of all gradients and the clipping coefficient
  ln_forward   layer norm of rows, optionally of the sum with a residual stream
  ln_backward  its gradients: of the rows, of weight and bias

8-bit states stand in blocks of 256 elements, each with two scales, the largest |m| and the largest v of the block.  m is held
as the nearest float8 e4m3 of 256 m / scale; v as eight bits c of an unsigned float with five bits of exponent and three of
mantissa, the float whose bits are c << 20 times 2^96 times the scale (nearest, ties to even, never 0 for a v above 0).  Scales
below 2^-126 count as 0, and so do the blocks.
"""
import math
import random

import numpy as np
import torch

own = False

BLOCK = 256
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
WIDTH = {"f32": 4, "bf16": 2, "f16": 2, "": 0}
ALPHA, BETA1, BETA2, EPS, DECAY, STEP = 1e-3, 0.9, 0.999, 1e-8, 0.1, 10


# ------------------------------------------------------------------------------------------ the tensors of a model

def _resnet_sizes(blocks, wide):
    sizes, inplanes, out = [(64 * 147, True), (64, False), (64, False)], 64, 4 if wide else 1
    for planes, count in zip((64, 128, 256, 512), blocks):
        for b in range(count):
            shapes = [planes * inplanes, planes * planes * 9, planes * planes * 4] if wide else \
                [planes * inplanes * 9, planes * planes * 9]
            for n, width in zip(shapes, [planes, planes, planes * 4] if wide else [planes, planes]):
                sizes += [(n, True), (width, False), (width, False)]
            if b == 0 and (wide or inplanes != planes):
                sizes += [(planes * out * inplanes, True), (planes * out, False), (planes * out, False)]
            inplanes = planes * out
    return sizes + [(1000 * inplanes, True), (1000, False)]


def _transformer_sizes(layers=48, hidden=1600, vocab=50257, positions=1024):
    h = hidden
    layer = [(h, False), (h, False), (3 * h * h, True), (3 * h, False), (h * h, True), (h, False), (h, False), (h, False),
             (4 * h * h, True), (4 * h, False), (4 * h * h, True), (h, False)]
    return [(vocab * h, True), (positions * h, True)] + layer * layers + [(h, False), (h, False)]


def _spread_sizes(d, count, seed):
    """`count` tensors of about d elements in all, sizes over four decades, odd ones among them; every third takes no decay."""
    share = 10.0 ** np.random.default_rng(seed).uniform(0.0, 4.0, count)
    return [(max(1, int(d * x)), i % 3 != 2) for i, x in enumerate(share / share.sum())]


def _tensors(case):
    """[(elements, whether weight decay applies)]"""
    model = case["model"]
    if model == "resnet18":
        return _resnet_sizes((2, 2, 2, 2), False)
    if model == "resnet50":
        return _resnet_sizes((3, 4, 6, 3), True)
    if model == "transformer":
        return _transformer_sizes()
    return _spread_sizes(case["d"], case["count"], case["layout"])


def _elements(case):
    return sum(n for n, _ in _tensors(case))


# ------------------------------------------------------------------------------------------ cases

def _step(path, model, *, d=0, count=0, layout=0, grad="f32", copy="", clip=False):
    return {"path": path, "model": model, "d": d, "count": count, "layout": layout, "grad": grad, "copy": copy, "clip": clip}


def _norm(path, rows, hidden, *, type="bf16", weights="f32", affine=2, stream=False, pad=0):
    return {"path": path, "rows": rows, "hidden": hidden, "type": type, "weights": weights, "affine": affine,
            "stream": stream, "pad": pad}


def listed():
    named = {
        # Toy problems and convergence runs: a step is launches and latency.
        "adamw_small": _step("adamw", "spread", d=65_537, count=6, layout=1, clip=True),
        # ResNet-50's 161 tensors behind a clipped norm, gradients as the decoder averages them, in 32 bits.
        "adamw_resnet50": _step("adamw", "resnet50", clip=True),
        # The 1.5 B transformer in mixed precision: gradients and the weights that the model computes with in bfloat16.
        "adamw_transformer": _step("adamw", "transformer", grad="bf16", copy="bf16", clip=True),
        # States in 8 bits: a small convolutional model, and the transformer, which they are there for.
        "adamw_coded_resnet18": _step("adamw_coded", "resnet18"),
        "adamw_coded_transformer": _step("adamw_coded", "transformer", grad="bf16", copy="bf16"),
        # The norm by itself, as it is logged and as a schedule of several optimizers shares it.
        "norm_transformer": _step("norm", "transformer"),
        # One token while text is generated: one row.
        "ln_forward_token": _norm("ln_forward", 1, 1600),
        # Eight sequences of 1024 positions through the transformer's width: between two blocks, with the residual stream, and back.
        "ln_forward_1600": _norm("ln_forward", 8192, 1600, stream=True),
        "ln_backward_1600": _norm("ln_backward", 8192, 1600, stream=True),
        # Widths that fit nothing: odd rows that are views into wider ones, weights in 16 bits too.
        "ln_backward_ragged": _norm("ln_backward", 5003, 1001, type="f16", weights="f16", pad=3),
        # The widest rows in 32 bits, and a long batch of wide rows in 16.
        "ln_forward_wide": _norm("ln_forward", 8192, 12288, type="f32"),
        "ln_backward_wide": _norm("ln_backward", 32768, 8192),
    }
    return [dict(c, name=n) for n, c in named.items()]


def _spread(rng, lo, hi):
    n = int(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.99))))
    n = min(hi, n | 1 if rng.random() < 0.4 else n)
    return n if n != 3072 else 3071


def draw(rng):
    path = rng.choice(["adamw", "adamw", "adamw_coded", "adamw_coded", "norm", "ln_forward", "ln_forward", "ln_backward",
                       "ln_backward"])
    if path.startswith("ln"):
        hidden = _spread(rng, 16, 16384)
        rows = _spread(rng, 1, min(65536, (1 << 27) // hidden))
        kind = rng.choice(["bf16", "bf16", "f16", "f32"])
        return _norm(path, rows, hidden, type=kind, weights=rng.choice(["f32", kind]), affine=rng.choice([2, 2, 2, 1, 0]),
                     stream=rng.random() < 0.5, pad=rng.choice([0, 0, 1, 8]))
    count = _spread(rng, 1, 300)
    d = _spread(rng, max(4096, 32 * count), 1 << 28)
    return _step(path, "spread", d=d, count=count, layout=rng.randrange(1000), grad=rng.choice(["f32", "f32", "bf16", "f16"]),
                 copy=rng.choice(["", "", "bf16", "f16"]) if path != "norm" else "", clip=path == "adamw" and rng.random() < 0.5)


# ------------------------------------------------------------------------------------------ inputs

def _flat(sizes, pad):
    """Where each tensor begins in a flat vector in which it takes a multiple of `pad`, and the vector's length."""
    starts, at = [], 0
    for n, _ in sizes:
        starts.append(at)
        at += -(-n // pad) * pad
    return starts, at


def _views(flat, starts, sizes):
    return [flat[o:o + n] for o, (n, _) in zip(starts, sizes)]


def _prepare_step(case, seed):
    """Weights, gradients and states after some steps.  The scale of a tensor's gradients is its own, over four decades; half
    the rows of the first tensor (an embedding) see no gradient in this step, and half of those never saw one."""
    dev = torch.device("cuda")
    coded, sizes = case["path"] == "adamw_coded", _tensors(case)
    starts, d = _flat(sizes, BLOCK if coded else 1)         # blocks of states begin with their tensor
    g = torch.Generator(device=dev).manual_seed(seed)
    rnd = lambda: torch.empty(d, dtype=torch.float32, device=dev).normal_(generator=g)  # noqa: E731
    sigma = 10.0 ** np.random.default_rng(seed).uniform(-5.0, -1.0, len(sizes))
    lengths = np.diff(np.append(starts, d))
    scale = torch.from_numpy(sigma.astype(np.float32)).to(dev).repeat_interleave(
        torch.from_numpy(lengths).to(dev), output_size=d)
    first, row = sizes[0][0], 512
    quiet = torch.rand(-(-first // row), generator=g, device=dev).repeat_interleave(row)[:first]
    live = None
    if coded:                                               # the flat vectors' gaps hold zeros, as a model's do
        live = torch.zeros(d, dtype=torch.bool, device=dev)
        for x in _views(live, starts, sizes):
            x.fill_(True)
    grad = rnd().mul_(scale)
    grad[:first].mul_(quiet >= 0.5)
    if live is not None:
        grad.mul_(live)
    grad = grad.to(TYPES[case["grad"]])
    st = {"case": case, "grads": _views(grad, starts, sizes), "flat_grad": grad,
          "max_norm": 0.7 * float(np.sqrt((sigma ** 2 * [n for n, _ in sizes]).sum()))}
    if case["path"] == "norm":
        _norm_workspace(st, dev)
        return st
    w = rnd().mul_(0.02)
    m = rnd().mul_(0.3).mul_(scale)
    v = rnd().square_().add_(0.2).mul_(scale).mul_(scale)
    never = quiet < 0.25
    m[:first].masked_fill_(never, 0.0)
    v[:first].masked_fill_(never, 0.0)
    if live is not None:
        for x in (w, m, v):
            x.mul_(live)
    del scale
    decay = [DECAY if heavy else 0.0 for _, heavy in sizes]
    st |= {"flat_w": w, "w": _views(w, starts, sizes), "decay": decay, "lengths": torch.from_numpy(lengths).to(dev)}
    if case["copy"]:
        copy = torch.empty(d, dtype=TYPES[case["copy"]], device=dev)
        if live is not None:
            copy.zero_()
        st |= {"flat_copy": copy, "copies": _views(copy, starts, sizes)}
    if coded:
        codes_m, codes_v, scales = _to_codes(m, v)
        blocks = [(o // BLOCK, -(-n // BLOCK)) for o, (n, _) in zip(starts, sizes)]
        st |= {"flat_m": codes_m, "flat_v": codes_v, "flat_scales": scales, "m": _views(codes_m, starts, sizes),
               "v": _views(codes_v, starts, sizes), "scales": [scales[2 * b:2 * (b + k)] for b, k in blocks],
               "coefficient": torch.full((1,), 0.5, dtype=torch.float32, device=dev),
               "values_m": torch.empty(d, dtype=torch.float32, device=dev),
               "values_v": torch.empty(d, dtype=torch.float32, device=dev)}
    else:
        st |= {"flat_m": m, "flat_v": v, "m": _views(m, starts, sizes), "v": _views(v, starts, sizes)}
        if case["clip"]:
            _norm_workspace(st, dev)
    return st


def _norm_workspace(st, dev):
    """What a program keeps for the norm: 64 KiB of scratch and the two numbers."""
    st["workspace"] = torch.empty(1 << 16, dtype=torch.uint8, device=dev)
    st["norm"] = torch.empty(2, dtype=torch.float32, device=dev)


def _prepare_rows(case, seed):
    dev = torch.device("cuda")
    rows, hidden, kind, wkind = case["rows"], case["hidden"], TYPES[case["type"]], TYPES[case["weights"]]
    g = torch.Generator(device=dev).manual_seed(seed)

    def rows_of(scale, shift=0.0):
        x = torch.empty(rows, hidden + case["pad"], dtype=torch.float32, device=dev).normal_(generator=g).mul_(scale)
        if shift:
            x.add_(shift * torch.randn(rows, 1, generator=g, device=dev))
        return x.to(kind)[:, :hidden]

    vector = lambda at, scale: (at + scale * torch.randn(hidden, generator=g, device=dev)).to(wkind)  # noqa: E731
    empty = lambda: torch.empty(rows, hidden, dtype=kind, device=dev)  # noqa: E731
    st = {"case": case, "eps": 1e-5, "x": rows_of(1.5, 0.7), "weight": vector(1.0, 0.2) if case["affine"] else None,
          "bias": vector(0.0, 0.2) if case["affine"] == 2 else None,
          "mean": torch.empty(rows, dtype=torch.float32, device=dev), "rstd": torch.empty(rows, dtype=torch.float32, device=dev)}
    if case["path"] == "ln_forward":
        st |= {"residual": rows_of(0.5) if case["stream"] else None, "total": empty() if case["stream"] else None, "y": empty()}
        return st
    x = st["x"].double() if rows * hidden < 1 << 22 else st["x"].float()
    st["mean"].copy_(x.mean(1))
    st["rstd"].copy_((x.var(1, correction=0) + st["eps"]).rsqrt())
    st |= {"dy": rows_of(0.1), "add": rows_of(0.1) if case["stream"] else None, "dx": empty(),
           "dweight": torch.empty_like(st["weight"]) if case["affine"] else None,
           "dbias": torch.empty_like(st["bias"]) if case["affine"] == 2 else None,
           "workspace": torch.empty(8 * hidden * min(rows, 1024), dtype=torch.uint8, device=dev)}
    return st


def prepare(case, seed):
    return _prepare_rows(case, seed) if case["path"].startswith("ln") else _prepare_step(case, seed)


# ------------------------------------------------------------------------------------------ one pass: plain form

def _from_codes(codes_m, codes_v, scales):
    a = scales.view(-1, 2, 1)
    m = codes_m.view(-1, BLOCK).float() * (a[:, 0] * 2.0 ** -8)
    v = (codes_v.view(-1, BLOCK).to(torch.int32) << 20).view(torch.float32) * 2.0 ** 96 * a[:, 1]
    return m.view(-1), v.view(-1)


def _to_codes(m, v):
    m, v = m.view(-1, BLOCK), v.view(-1, BLOCK)
    a = torch.stack([m.abs().amax(1), v.amax(1)], 1)
    a = torch.where(a < 2.0 ** -126, torch.zeros_like(a), a)
    inv = torch.where(a > 0.0, torch.ones_like(a) / a, torch.zeros_like(a))
    codes_m = (m * inv[:, :1] * 256.0).to(torch.float8_e4m3fn)
    bits = (v * inv[:, 1:] * 2.0 ** -96).view(torch.int32)
    codes_v = (bits + 0x7FFFF + ((bits >> 20) & 1)) >> 20
    codes_v = torch.maximum(codes_v, ((v > 0.0) & (a[:, 1:] > 0.0)).to(torch.int32)).to(torch.uint8)
    return codes_m.view(-1), codes_v.view(-1), a.view(-1)


def _plain_norm(st):
    norm = st["flat_grad"].float().square().sum().sqrt()
    c = torch.where(norm > st["max_norm"], st["max_norm"] / norm, torch.ones_like(norm))
    return torch.stack([norm, c])


def _plain_step(st, m, v, coefficient):
    """New weights and moments; the weights are moved in place."""
    w, g = st["flat_w"], st["flat_grad"].float()
    if coefficient is not None:
        g = g * coefficient
    m = m * BETA1 + g * (1.0 - BETA1)
    v = v * BETA2 + g * g * (1.0 - BETA2)
    del g
    u = m / (v.sqrt() * (1.0 / math.sqrt(1.0 - BETA2 ** STEP)) + EPS)
    keep = torch.tensor([1.0 - ALPHA * x for x in st["decay"]], dtype=torch.float32, device=w.device)
    keep = keep.repeat_interleave(st["lengths"], output_size=w.numel())
    w.copy_(w * keep - u * (ALPHA / (1.0 - BETA1 ** STEP)))
    if "flat_copy" in st:
        st["flat_copy"].copy_(w)
    return m, v


def _plain(st):
    case = st["case"]
    if case["path"] == "norm":
        return _plain_norm(st)
    if case["path"] == "adamw":
        norm = _plain_norm(st) if case["clip"] else None
        m, v = _plain_step(st, st["flat_m"], st["flat_v"], None if norm is None else norm[1])
        st["flat_m"].copy_(m)
        st["flat_v"].copy_(v)
        return _step_outputs(st, st["flat_m"], st["flat_v"], norm)
    if case["path"] == "adamw_coded":
        m, v = _plain_step(st, *_from_codes(st["flat_m"], st["flat_v"], st["flat_scales"]), st["coefficient"])
        codes = _to_codes(m, v)
        del m, v
        for to, x in zip(("flat_m", "flat_v", "flat_scales"), codes):
            st[to].copy_(x)
        return _step_outputs(st, *_from_codes(*codes), None)
    x = st["x"].float()
    weight = st["weight"].float() if st["weight"] is not None else 1.0
    if case["path"] == "ln_forward":
        total = None
        if st["residual"] is not None:
            total = (x + st["residual"].float()).to(st["x"].dtype)
            x = total.float()
        mean = x.mean(1, keepdim=True)
        x = x - mean
        rstd = (x.square().mean(1, keepdim=True) + st["eps"]).rsqrt()
        y = x * rstd * weight
        if st["bias"] is not None:
            y = y + st["bias"].float()
        return {"y": y.to(st["x"].dtype), "total": total, "mean": mean.view(-1), "rstd": rstd.view(-1)}
    xhat = (x - st["mean"][:, None]) * st["rstd"][:, None]
    dy = st["dy"].float()
    dw = (dy * xhat).sum(0).to(st["weight"].dtype) if st["weight"] is not None else None
    db = dy.sum(0).to(st["bias"].dtype) if st["bias"] is not None else None
    dy = dy * weight
    dx = (dy - dy.mean(1, keepdim=True) - xhat * (dy * xhat).mean(1, keepdim=True)) * st["rstd"][:, None]
    if st["add"] is not None:
        dx = dx + st["add"].float()
    return {"dx": dx.to(st["x"].dtype), "dweight": dw, "dbias": db}


def _step_outputs(st, m, v, norm):
    return {"w": st["flat_w"], "copy": st.get("flat_copy"), "m": m, "v": v, "norm": norm}


# ------------------------------------------------------------------------------------------ one pass: the framework's kernels

def _framework(st):
    import paper_1908_06077_amd as nuq
    case = st["case"]
    path = case["path"]
    if path == "ln_forward":
        nuq.nuq_layer_norm_forward(st["x"], st["residual"], st["weight"], st["bias"], st["eps"], st["total"], st["y"],
                                   st["mean"], st["rstd"])
        return {"y": st["y"], "total": st["total"], "mean": st["mean"], "rstd": st["rstd"]}
    if path == "ln_backward":
        nuq.nuq_layer_norm_backward(st["dy"], st["x"], st["weight"], st["mean"], st["rstd"], st["add"], st["dx"],
                                    st["dweight"], st["dbias"], st["workspace"])
        return {"dx": st["dx"], "dweight": st["dweight"], "dbias": st["dbias"]}
    norm = coefficient = None
    if path == "norm" or case["clip"]:
        norm = st["norm"]
        nuq.nuq_gradient_norm(st["grads"], st["max_norm"], st["workspace"], norm)
        coefficient = norm[1:]
        if path == "norm":
            return norm
    hyper = (st["decay"], ALPHA, BETA1, BETA2, EPS, STEP)
    if path == "adamw":
        nuq.nuq_adamw_step(st["w"], st["grads"], st["m"], st["v"], *hyper, coefficient, st.get("copies"))
        return _step_outputs(st, st["flat_m"], st["flat_v"], norm)
    nuq.nuq_adamw_step_coded(st["w"], st["grads"], st["m"], st["v"], st["scales"], *hyper, st["coefficient"], st.get("copies"))
    nuq.nuq_adamw_state_values(st["flat_m"], st["flat_v"], st["flat_scales"], st["values_m"], st["values_v"])
    return _step_outputs(st, st["values_m"], st["values_v"], None)


def run(state):
    return _framework(state) if own else _plain(state)


# ------------------------------------------------------------------------------------------ what a pass cannot do without

def work(case):
    path = case["path"]
    if path.startswith("ln"):
        rows, hidden, wide = case["rows"], case["hidden"], WIDTH[case["type"]]
        n, vectors = rows * hidden, case["affine"] * hidden * WIDTH[case["weights"]]
        if path == "ln_forward":
            return {"bytes": n * wide * (4 if case["stream"] else 2) + vectors + 8 * rows, "flops": 9 * n}
        weight = hidden * WIDTH[case["weights"]] * min(1, case["affine"])
        return {"bytes": n * wide * (4 if case["stream"] else 3) + weight + vectors + 8 * rows, "flops": 16 * n}
    d, grad = _elements(case), WIDTH[case["grad"]]
    if path == "norm":
        return {"bytes": d * grad + 8, "flops": 2 * d}
    if path == "adamw":
        return {"bytes": d * (24 + grad + WIDTH[case["copy"]]), "flops": (18 if case["clip"] else 15) * d}
    # weights, gradient, codes in and out, scales in and out, the values that the codes stand for
    return {"bytes": d * (8 + grad + 4 + WIDTH[case["copy"]] + 8) + 16 * -(-d // BLOCK), "flops": 34 * d}


# ------------------------------------------------------------------------------------------ the definition in 64 bits

def _nearest(y, fraction_bits, lowest):
    """The nearest float with so many bits of fraction and 2^lowest as its least normal number, ties to even."""
    e = torch.frexp(y.abs())[1] - 1
    step = torch.ldexp(torch.ones_like(y), e.clamp(min=lowest) - fraction_bits)
    return torch.round(y / step) * step


def _exact_codes(m, v):
    """The values that the codes of moments in 64 bits stand for."""
    m, v = m.view(-1, BLOCK), v.view(-1, BLOCK)
    top_m, top_v = m.abs().amax(1, keepdim=True), v.amax(1, keepdim=True)
    one = torch.ones_like(top_m)
    top_m, top_v = (torch.where(t < 2.0 ** -126, 0.0 * one, t) for t in (top_m, top_v))
    div_m, div_v = (torch.where(t > 0.0, t, one) for t in (top_m, top_v))
    held_m = _nearest(m / div_m * 256.0, 3, -6) / 256.0 * top_m
    held_v = _nearest(v / div_v * 2.0 ** 31, 3, 1)          # least normal number 2^1, steps of 1/4 below it
    held_v = torch.where((v > 0.0) & (held_v == 0.0), 0.25 * torch.ones_like(v), held_v) * 2.0 ** -31 * top_v
    return held_m.view(-1), held_v.view(-1)


def _exact_step(st):
    case = st["case"]
    coded = case["path"] == "adamw_coded"
    d, dev, norm, c = st["flat_grad"].numel(), st["flat_grad"].device, None, None
    part = 1 << 26
    if case["path"] == "norm" or case["clip"]:
        total = torch.zeros((), dtype=torch.float64, device=dev)
        for lo in range(0, d, part):
            total += st["flat_grad"][lo:lo + part].double().square().sum()
        root = total.sqrt()
        norm = torch.stack([root, (st["max_norm"] / root).clamp(max=1.0)])
        c = norm[1]
    if case["path"] == "norm":
        return norm
    if coded:
        c = st["coefficient"].double()
    keep = torch.tensor([1.0 - ALPHA * x for x in st["decay"]], dtype=torch.float64, device=dev)
    ends = st["lengths"].cumsum(0)
    out = {k: torch.empty(d, dtype=torch.float64, device=dev) for k in ("w", "m", "v")}
    for lo in range(0, d, part):
        hi = min(d, lo + part)
        g = st["flat_grad"][lo:hi].double()
        if c is not None:
            g = c * g
        if coded:
            a = st["flat_scales"].double().view(-1, 2)[lo // BLOCK:hi // BLOCK, :, None]
            m = (st["flat_m"][lo:hi].float().double().view(-1, BLOCK) / 256.0 * a[:, 0]).view(-1)
            code = st["flat_v"][lo:hi].long()
            e, f = code // 8, code % 8
            unit = torch.where(e > 0, (8 + f).double() * 2.0 ** (e - 1).clamp(min=0).double(), f.double())
            v = (unit.view(-1, BLOCK) * 2.0 ** -33 * a[:, 1]).view(-1)
        else:
            m, v = st["flat_m"][lo:hi].double(), st["flat_v"][lo:hi].double()
        m = BETA1 * m + (1.0 - BETA1) * g
        v = BETA2 * v + (1.0 - BETA2) * g ** 2
        of = torch.searchsorted(ends, torch.arange(lo, hi, device=dev), right=True)
        mhat, vhat = m / (1.0 - BETA1 ** STEP), v / (1.0 - BETA2 ** STEP)
        out["w"][lo:hi] = st["flat_w"][lo:hi].double() * keep[of] - ALPHA * mhat / (vhat ** 0.5 + EPS)
        out["m"][lo:hi], out["v"][lo:hi] = _exact_codes(m, v) if coded else (m, v)
    return {"w": out["w"], "copy": out["w"] if case["copy"] else None, "m": out["m"], "v": out["v"], "norm": norm}


def _exact_rows(st):
    case = st["case"]
    x = st["x"].double()
    hidden = case["hidden"]
    weight = torch.ones(hidden, dtype=torch.float64, device=x.device) if st["weight"] is None else st["weight"].double()
    if case["path"] == "ln_forward":
        total = None
        if st["residual"] is not None:
            total = x + st["residual"].double()
            x = total.to(st["x"].dtype).double()             # the sum is what the stream holds: rounded to its type
        mean = x.sum(1) / hidden
        var = ((x - mean[:, None]) ** 2).sum(1) / hidden
        rstd = 1.0 / (var + st["eps"]) ** 0.5
        y = (x - mean[:, None]) * (rstd[:, None] * weight)
        return {"y": y if st["bias"] is None else y + st["bias"].double(), "total": total, "mean": mean, "rstd": rstd}
    n, rstd = (x - st["mean"].double()[:, None]), st["rstd"].double()[:, None]
    n = n * rstd
    dy = st["dy"].double()
    dweight = (dy * n).sum(0) if st["weight"] is not None else None
    dbias = dy.sum(0) if st["bias"] is not None else None
    dn = dy * weight
    dx = rstd / hidden * (hidden * dn - dn.sum(1, keepdim=True) - n * (dn * n).sum(1, keepdim=True))
    return {"dx": dx if st["add"] is None else dx + st["add"].double(), "dweight": dweight, "dbias": dbias}


def exact(case, seed):
    st = prepare(case, seed)
    return _exact_rows(st) if case["path"].startswith("ln") else _exact_step(st)


if __name__ == "__main__":
    for c in listed() + [draw(random.Random(k)) for k in range(6)]:
        print(c, work(c))
