"""The operators between and behind a transformer's products as measurable cases: one case is one pass through one of them at one size.

Paths (one pass each):
  dropout      y = x kept with the chance 1 - p and scaled, optionally added to a residual stream; the mask comes from a counter
  rn_forward   the seam of two blocks: a norm of the branch, gate, dropout, scales and the residual sum, and the sum's norm
  rn_backward  its gradients: of branch and stream, of the norms' weights and the gate
  ce_forward   softmax cross entropy of the rows x against the vocabulary's weights, loss and log-sum-exp per row, and their mean
  ce_backward  its gradients: of rows and weights

The draws.  Element (r, c) of rows: z = seed + step * 0xD1342543DE82EF95 + (r + 1) * 0x9E3779B97F4A7C15 modulo 2^64 goes through
z = (z ^ z >> 30) * 0xBF58476D1CE4E5B9, z = (z ^ z >> 27) * 0x94D049BB133111EB, z ^= z >> 31; with its lower half k0 and its upper
half k1, x = (k0 + c) * 0x9E3779B1, x = (x ^ x >> 15 ^ k1) * 0x85EBCA6B, x ^= x >> 16 modulo 2^32, and the element is kept where
x >> 8 is at least T = p 2^24 rounded; what is kept is multiplied with 2^24 / (2^24 - T).
"""
import math
import random

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
WIDTH = {"f32": 4, "bf16": 2, "f16": 2}
IGNORED = -100
EPS = 1e-5


# ------------------------------------------------------------------------------------------ cases

def _dropout(rows, hidden, *, type="bf16", p=0.1, stream=False, pad=0):
    return {"path": "dropout", "rows": rows, "hidden": hidden, "type": type, "p": p, "stream": stream, "pad": pad}


def _seam(path, rows, hidden, *, type="bf16", weights="f32", inner="layer", outer="layer", bias=True, gate=True, scale=1.0,
          residual_scale=1.0, p=0.0, pad=0):
    return {"path": path, "rows": rows, "hidden": hidden, "type": type, "weights": weights, "inner": inner, "outer": outer,
            "bias": bias, "gate": gate, "scale": scale, "residual_scale": residual_scale, "p": p, "pad": pad}


def _loss(path, rows, hidden, vocab, *, type="bf16", smoothing=0.0, ignored=0.1, pad=0):
    return {"path": path, "rows": rows, "hidden": hidden, "vocab": vocab, "type": type, "smoothing": smoothing, "ignored": ignored,
            "pad": pad}


def listed():
    named = {
        # The embeddings of one short sequence while a model is tuned: a launch.
        "dropout_small": _dropout(128, 1600),
        # A branch of a wide layer over sixteen sequences of 1024 positions, added to the stream on the way.
        "dropout_large": _dropout(16384, 6400, stream=True),
        # A width that fits nothing, rows that are views into wider ones, in 32 bits.
        "dropout_ragged": _dropout(5003, 1001, type="f32", p=0.25, pad=3),
        # One token while text is generated: the sum and the next block's norm, nothing dropped.
        "rn_forward_token": _seam("rn_forward", 1, 1600, inner="none", scale=0.5),
        # Eight sequences of 1024 positions through the transformer's width, a norm on either side of the seam, and back.
        "rn_forward_1600": _seam("rn_forward", 8192, 1600, p=0.1),
        "rn_backward_1600": _seam("rn_backward", 8192, 1600, p=0.1),
        # Odd rows that are views into wider ones, weights in 16 bits too, both norms without mean and bias.
        "rn_backward_ragged": _seam("rn_backward", 5003, 1001, type="f16", weights="f16", inner="rms", outer="rms", bias=False, pad=3),
        # A long batch of wide rows.
        "rn_backward_wide": _seam("rn_backward", 16384, 8192, inner="rms", outer="rms", bias=False, residual_scale=0.7),
        # Scoring one token against the transformer's whole vocabulary: its weights are read once.
        "ce_forward_token": _loss("ce_forward", 1, 1600, 50257, ignored=0.0),
        # The training step of eight sequences of 1024 positions: the loss, and its gradients.
        "ce_forward_1600": _loss("ce_forward", 8192, 1600, 50257),
        "ce_backward_1600": _loss("ce_backward", 8192, 1600, 50257),
        # Nothing fits a tile: odd rows, widths and vocabulary, views, smoothed targets.
        "ce_backward_ragged": _loss("ce_backward", 1003, 1001, 10007, type="f16", smoothing=0.1, pad=3),
    }
    return [dict(c, name=n) for n, c in named.items()]


def _spread(rng, lo, hi):
    n = int(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.99))))
    return min(hi, n | 1 if rng.random() < 0.4 else n)


def draw(rng):
    path = rng.choice(["dropout", "dropout", "rn_forward", "rn_forward", "rn_backward", "rn_backward", "ce_forward", "ce_forward",
                       "ce_backward", "ce_backward"])
    kind, pad = rng.choice(["bf16", "bf16", "f16", "f32"]), rng.choice([0, 0, 1, 8])
    if path == "dropout":
        hidden = _spread(rng, 1, 65536)
        return _dropout(_spread(rng, 1, min(1 << 20, (1 << 26) // hidden)), hidden, type=kind, p=rng.choice([0.0, 0.1, 0.5]),
                        stream=rng.random() < 0.5, pad=pad)
    if path.startswith("rn"):
        hidden = _spread(rng, 16, 16384)
        inner, outer = rng.choice([("layer", "layer"), ("rms", "rms"), ("none", "layer"), ("none", "rms"), ("rms", "none")])
        return _seam(path, _spread(rng, 1, min(65536, (1 << 26) // hidden)), hidden, type=kind, weights=rng.choice(["f32", kind]),
                     inner=inner, outer=outer, bias=rng.random() < 0.5, gate=rng.random() < 0.5, scale=rng.choice([1.0, 0.5]),
                     residual_scale=rng.choice([1.0, 0.7]), p=rng.choice([0.0, 0.1, 0.3]), pad=pad)
    hidden, vocab = _spread(rng, 32, 4096), _spread(rng, 256, 131072)
    rows = _spread(rng, 1, min(16384, (1 << 28) // vocab))
    return _loss(path, rows, hidden, vocab, type=kind, smoothing=rng.choice([0.0, 0.0, 0.1]), ignored=rng.choice([0.0, 0.1, 0.5]),
                 pad=pad)


# ------------------------------------------------------------------------------------------ inputs

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _rows(case, g, scale, shift=0.0):
    """Rows at a stride that is `pad` elements longer than they are."""
    x = torch.empty(case["rows"], case["hidden"] + case["pad"], dtype=torch.float32, device="cuda").normal_(generator=g).mul_(scale)
    if shift:
        x.add_(shift * torch.randn(case["rows"], 1, generator=g, device="cuda"))
    return x.to(TYPES[case["type"]])[:, :case["hidden"]]


def _like(case):
    return torch.empty(case["rows"], case["hidden"], dtype=TYPES[case["type"]], device="cuda")


def _prepare_dropout(case, seed):
    g = _generator(seed)
    return {"case": case, "seed": 977 * seed + 5, "step": torch.full((1,), seed % 1000, dtype=torch.int64, device="cuda"),
            "x": _rows(case, g, 1.0), "residual": _rows(case, g, 2.0) if case["stream"] else None, "y": _like(case)}


def _prepare_seam(case, seed):
    g = _generator(seed)
    wide, rows, hidden = TYPES[case["weights"]], case["rows"], case["hidden"]
    vector = lambda at, s: (at + s * torch.randn(hidden, generator=g, device="cuda")).to(wide)  # noqa: E731
    st = {"case": case, "seed": 977 * seed + 5, "step": torch.full((1,), seed % 1000, dtype=torch.int64, device="cuda"),
          "x": _rows(case, g, 1.5, 0.3), "residual": _rows(case, g, 2.0, 0.2),
          "w1": vector(1.0, 0.2) if case["inner"] != "none" else None,
          "b1": vector(0.0, 0.2) if case["inner"] != "none" and case["bias"] else None,
          "gate": vector(0.3, 0.1) if case["gate"] else None,
          "w2": vector(1.0, 0.2) if case["outer"] != "none" else None,
          "b2": vector(0.0, 0.2) if case["outer"] != "none" and case["bias"] else None,
          "stats": torch.zeros(4, rows, dtype=torch.float32, device="cuda")}
    if case["path"] == "rn_forward":
        return st | {"total": _like(case), "y": _like(case) if case["outer"] != "none" else None}
    forward = _plain_seam(st)
    st["total"] = forward["total"]
    for k, name in enumerate(STATS):
        if forward[name] is not None:
            st["stats"][k].copy_(forward[name])
    empty = lambda v: None if v is None else torch.empty_like(v)  # noqa: E731
    return st | {"dy": _rows(case, g, 0.1) if case["outer"] != "none" else None, "dtotal": _rows(case, g, 0.1), "dx": _like(case),
                 "dresidual": _like(case), "dw1": empty(st["w1"]), "db1": empty(st["b1"]), "dgate": empty(st["gate"]),
                 "dw2": empty(st["w2"]), "db2": empty(st["b2"]),
                 # what a program keeps for it: five sums of the columns for each of up to 1024 parts of the rows, two numbers per row
                 "workspace": torch.empty(20 * hidden * min(rows, 1024) + 16 * rows + 64, dtype=torch.uint8, device="cuda")}


def _prepare_loss(case, seed):
    """Logits of a model that has learned something: 2 in standard deviation, the target's 6 above, a part of the rows padding."""
    g = _generator(seed)
    rows, hidden, vocab, kind = case["rows"], case["hidden"], case["vocab"], TYPES[case["type"]]
    w = torch.empty(vocab, hidden + case["pad"], dtype=torch.float32, device="cuda").normal_(generator=g).mul_(2.0 / math.sqrt(hidden))
    target = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    x = torch.empty(rows, hidden + case["pad"], dtype=torch.float32, device="cuda").normal_(generator=g)
    x = x.add_(w[target], alpha=1.5).to(kind)[:, :hidden]
    if case["ignored"]:
        target[torch.rand(rows, generator=g, device="cuda") < case["ignored"]] = IGNORED
    st = {"case": case, "x": x, "weight": w.to(kind)[:, :hidden], "target": target,
          "workspace": torch.empty(_loss_workspace(case), dtype=torch.uint8, device="cuda")}
    del w
    if case["path"] == "ce_forward":
        return st | {"loss": torch.empty(rows, device="cuda"), "lse": torch.empty(rows, device="cuda"),
                     "mean": torch.empty(2, device="cuda")}
    lse = torch.cat([torch.logsumexp(x[at:at + 4096].float() @ st["weight"].float().t(), 1) for at in range(0, rows, 4096)])
    valid = (target != IGNORED).sum()
    mean = torch.stack([torch.zeros_like(valid, dtype=torch.float32), 1.0 / valid.clamp(min=1).float()])
    return st | {"lse": lse, "mean": mean, "grad": torch.full((1,), 1.0, device="cuda"), "dx": _like(case),
                 "dweight": torch.empty(vocab, hidden, dtype=kind, device="cuda")}


def _loss_workspace(case):
    """What a program keeps for the loss: forward some numbers per row and 128 entries of the vocabulary and room for rows that have to
    be laid out anew, backward besides a piece of the vocabulary at a time, at most 2 GiB of it."""
    rows, hidden, vocab, wide = (case[k] for k in ("rows", "hidden", "vocab", "type"))
    wide, up = WIDTH[wide], lambda n, m: -(-n // m) * m  # noqa: E731
    copies = (up(rows, 256) + up(vocab, 256)) * up(hidden, 64) * wide
    forward = 16 * up(rows, 256) * (up(vocab, 128) // 128) + 64 * up(rows, 256) + copies + (1 << 20)
    if case["path"] == "ce_forward":
        return forward
    return forward + copies + 4 * up(rows, 256) * up(hidden, 256) + min(2 << 30, 2 * wide * up(rows, 256) * up(vocab, 256)) + (1 << 22)


def prepare(case, seed):
    kind = case["path"][:2]
    return (_prepare_dropout if kind == "dr" else _prepare_seam if kind == "rn" else _prepare_loss)(case, seed)


# ------------------------------------------------------------------------------------------ one pass: plain form

STATS = ("mean1", "rstd1", "mean2", "rstd2")
M32 = 0xFFFFFFFF


def _signed(x):
    x &= 0xFFFFFFFFFFFFFFFF
    return x - (1 << 64) if x >> 63 else x


def _threshold(p):
    return math.floor(p * 2.0 ** 24 + 0.5)


def _plain_factors(st, rows, hidden):
    """The mask as factors in 32 bits: 0, or what is kept is multiplied with."""
    dev, top = st["x"].device, _threshold(st["case"]["p"])
    z = torch.arange(1, rows + 1, dtype=torch.int64, device=dev) * _signed(0x9E3779B97F4A7C15)
    z = z + (st["step"] * _signed(0xD1342543DE82EF95) + st["seed"])
    z = (z ^ ((z >> 30) & (1 << 34) - 1)) * _signed(0xBF58476D1CE4E5B9)
    z = (z ^ ((z >> 27) & (1 << 37) - 1)) * _signed(0x94D049BB133111EB)
    z = z ^ ((z >> 31) & (1 << 33) - 1)
    low, high = (z & M32)[:, None], ((z >> 32) & M32)[:, None]
    u = ((low + torch.arange(hidden, dtype=torch.int64, device=dev)) * 0x9E3779B1) & M32
    u = ((u ^ (u >> 15) ^ high) * 0x85EBCA6B) & M32
    u = (u ^ (u >> 16)) >> 8
    return (u >= top).float() * (2.0 ** 24 / (2 ** 24 - top))


def _plain_dropout(st):
    x = st["x"].float()
    if _threshold(st["case"]["p"]):
        x = x * _plain_factors(st, *x.shape)
    if st["residual"] is not None:
        x = x + st["residual"].float()
    return x.to(st["x"].dtype)


def _plain_norm(s, kind):
    """(normed rows, mean or none, rstd)"""
    mean = s.mean(1, keepdim=True) if kind == "layer" else None
    if mean is not None:
        s = s - mean
    rstd = (s.square().mean(1, keepdim=True) + EPS).rsqrt()
    return s * rstd, mean, rstd


def _affine(n, w, b):
    if w is not None:
        n = n * w.float()
    return n if b is None else n + b.float()


def _plain_seam(st):
    case = st["case"]
    s, mean1, rstd1 = st["x"].float(), None, None
    if case["inner"] != "none":
        s, mean1, rstd1 = _plain_norm(s, case["inner"])
        s = _affine(s, st["w1"], st["b1"])
    if st["gate"] is not None:
        s = s * st["gate"].float()
    if _threshold(case["p"]):
        s = s * _plain_factors(st, *s.shape)
    total = (st["residual"].float() * case["residual_scale"] + s * case["scale"]).to(st["x"].dtype)
    y, mean2, rstd2 = None, None, None
    if case["outer"] != "none":
        y, mean2, rstd2 = _plain_norm(total.float(), case["outer"])
        y = _affine(y, st["w2"], st["b2"]).to(st["x"].dtype)
    flat = lambda v: None if v is None else v.view(-1)  # noqa: E731
    return {"total": total, "y": y, "mean1": flat(mean1), "rstd1": flat(rstd1), "mean2": flat(mean2), "rstd2": flat(rstd2)}


def _plain_norm_gradient(d, n, rstd, kind):
    d = d - n * (d * n).mean(1, keepdim=True) - (d.mean(1, keepdim=True) if kind == "layer" else 0.0)
    return d * rstd[:, None]


def _plain_seam_gradients(st):
    case = st["case"]
    mean1, rstd1, mean2, rstd2 = st["stats"]
    to = lambda v, like: None if like is None else v.sum(0).to(like.dtype)  # noqa: E731
    dt, dw2, db2 = st["dtotal"].float(), None, None
    if case["outer"] != "none":
        n = st["total"].float()
        n = (n - mean2[:, None] if case["outer"] == "layer" else n) * rstd2[:, None]
        dy = st["dy"].float()
        dw2, db2 = to(dy * n, st["w2"]), to(dy, st["b2"])
        dt = dt + _plain_norm_gradient(dy * st["w2"].float(), n, rstd2, case["outer"])
    dresidual = (dt * case["residual_scale"]).to(st["x"].dtype)
    dt = dt * case["scale"]
    if _threshold(case["p"]):
        dt = dt * _plain_factors(st, *dt.shape)
    n = st["x"].float()
    if case["inner"] != "none":
        n = (n - mean1[:, None] if case["inner"] == "layer" else n) * rstd1[:, None]
    dgate = to(dt * _affine(n, st["w1"], st["b1"]), st["gate"])
    if st["gate"] is not None:
        dt = dt * st["gate"].float()
    dw1, db1 = to(dt * n, st["w1"]), to(dt, st["b1"])
    if case["inner"] != "none":
        dt = _plain_norm_gradient(dt * st["w1"].float(), n, rstd1, case["inner"])
    return {"dx": dt.to(st["x"].dtype), "dresidual": dresidual, "dw1": dw1, "db1": db1, "dgate": dgate, "dw2": dw2, "db2": db2}


def _plain_loss(st):
    case = st["case"]
    z = st["x"].float() @ st["weight"].float().t()
    top = z.amax(1, keepdim=True)
    lse = (z - top).exp().sum(1).log() + top[:, 0]
    valid = st["target"] != IGNORED
    loss = lse - (1.0 - case["smoothing"]) * z.gather(1, st["target"].clamp(min=0)[:, None])[:, 0] - case["smoothing"] * z.mean(1)
    loss = torch.where(valid, loss, torch.zeros_like(loss))
    part = 1.0 / valid.sum().clamp(min=1).float()
    return {"loss": loss, "lse": lse, "mean": torch.stack([loss.sum() * part, part])}


def _plain_loss_gradients(st):
    case = st["case"]
    x, w, valid = st["x"].float(), st["weight"].float(), st["target"] != IGNORED
    d = (x @ w.t() - st["lse"][:, None]).exp() - case["smoothing"] / case["vocab"]
    d.scatter_add_(1, st["target"].clamp(min=0)[:, None], torch.full_like(st["lse"], case["smoothing"] - 1.0)[:, None])
    d = d * torch.where(valid, st["grad"] * st["mean"][1], torch.zeros_like(st["lse"]))[:, None]
    return {"dx": (d @ w).to(st["x"].dtype), "dweight": (d.t() @ x).to(st["x"].dtype)}


def _plain(st):
    return {"dropout": _plain_dropout, "rn_forward": _plain_seam, "rn_backward": _plain_seam_gradients, "ce_forward": _plain_loss,
            "ce_backward": _plain_loss_gradients}[st["case"]["path"]](st)


# ------------------------------------------------------------------------------------------ one pass: the framework's kernels

def _framework(st):
    import paper_1908_06077_amd as nuq
    case = st["case"]
    path = case["path"]
    if path == "dropout":
        nuq.nuq_dropout(st["x"], st["residual"], case["p"], st["seed"], st["step"], st["y"])
        return st["y"]
    if path.startswith("rn"):
        kinds = {"none": nuq.NO_NORM, "layer": nuq.LAYER_NORM, "rms": nuq.RMS_NORM}
        inner, outer = kinds[case["inner"]], kinds[case["outer"]]
        numbers = (case["scale"], case["residual_scale"], case["p"], st["seed"], st["step"])
        if path == "rn_forward":
            nuq.nuq_residual_norm_forward(st["x"], st["residual"], inner, st["w1"], st["b1"], st["gate"], outer, st["w2"], st["b2"],
                                          EPS, *numbers, st["total"], st["y"], st["stats"])
            there = (case["inner"] == "layer", case["inner"] != "none", case["outer"] == "layer", case["outer"] != "none")
            return {"total": st["total"], "y": st["y"],
                    **{name: st["stats"][k] if is_there else None for k, (name, is_there) in enumerate(zip(STATS, there))}}
        nuq.nuq_residual_norm_backward(st["dy"], st["dtotal"], st["x"], st["total"], inner, st["w1"], st["b1"], st["gate"], outer,
                                       st["w2"], *numbers, st["stats"], st["dx"], st["dresidual"], st["dw1"], st["db1"], st["dgate"],
                                       st["dw2"], st["db2"], st["workspace"])
        return {k: st[k] for k in ("dx", "dresidual", "dw1", "db1", "dgate", "dw2", "db2")}
    if path == "ce_forward":
        nuq.nuq_linear_cross_entropy_forward(st["x"], st["weight"], st["target"], IGNORED, case["smoothing"], st["loss"], st["lse"],
                                             st["mean"], st["workspace"])
        return {k: st[k] for k in ("loss", "lse", "mean")}
    nuq.nuq_linear_cross_entropy_backward(st["x"], st["weight"], st["target"], IGNORED, case["smoothing"], st["lse"], st["grad"],
                                          st["mean"], st["dx"], st["dweight"], st["workspace"])
    return {k: st[k] for k in ("dx", "dweight")}


def run(state):
    return _framework(state) if own else _plain(state)


# ------------------------------------------------------------------------------------------ what a pass cannot do without

def work(case):
    path, rows, hidden, wide = case["path"], case["rows"], case["hidden"], WIDTH[case["type"]]
    n = rows * hidden
    if path == "dropout":
        return {"bytes": n * wide * (3 if case["stream"] else 2) + 8, "flops": 12 * n}
    if path.startswith("rn"):
        inner, outer = case["inner"] != "none", case["outer"] != "none"
        vectors = hidden * WIDTH[case["weights"]] * (case["gate"] + (inner + outer) * (1 + case["bias"]))
        numbers = 4 * rows * ((inner and 1 + (case["inner"] == "layer")) + (outer and 1 + (case["outer"] == "layer")))
        if path == "rn_forward":
            return {"bytes": n * wide * (3 + outer) + vectors + numbers, "flops": 22 * n}
        return {"bytes": n * wide * (4 + 2 * outer) + 2 * vectors + numbers, "flops": 44 * n}
    weights, product = case["vocab"] * hidden, 2 * n * case["vocab"]
    if path == "ce_forward":
        return {"bytes": wide * (n + weights) + 16 * rows + 8, "flops": product}
    return {"bytes": 2 * wide * (n + weights) + 12 * rows, "flops": 3 * product}


# ------------------------------------------------------------------------------------------ the definition in 64 bits

def _exact_kept(st, first, rows, hidden):
    """Which elements of `rows` rows from row `first` on are kept, as 0 and 1 in 64 bits."""
    mask, keys = (1 << 64) - 1, []
    begin = st["seed"] + int(st["step"].item()) * 0xD1342543DE82EF95
    for r in range(first, first + rows):
        z = (begin + (r + 1) * 0x9E3779B97F4A7C15) & mask
        z = ((z ^ z >> 30) * 0xBF58476D1CE4E5B9) & mask
        z = ((z ^ z >> 27) * 0x94D049BB133111EB) & mask
        keys.append(z ^ z >> 31)
    wrap = lambda v: v - (1 << 32) if v >> 31 else v  # noqa: E731
    vector = lambda vs: torch.tensor([wrap(v) for v in vs], dtype=torch.int32, device="cuda")[:, None]  # noqa: E731
    x = torch.arange(hidden, dtype=torch.int32, device="cuda")[None] + vector([k & M32 for k in keys])
    x = x * wrap(0x9E3779B1)                                # 32-bit products wrap
    x = (x ^ ((x >> 15) & 0x1FFFF) ^ vector([k >> 32 for k in keys])) * wrap(0x85EBCA6B)
    x = x ^ ((x >> 16) & 0xFFFF)
    return (((x >> 8) & 0xFFFFFF) >= _threshold(st["case"]["p"])).double()


def _in_parts(st, part, f):
    """f(first row, rows) over parts of the rows, its lists of results put together."""
    rows = st["x"].shape[0]
    found = [f(at, min(part, rows - at)) for at in range(0, rows, part)]
    return [None if c[0] is None else torch.cat(c) for c in zip(*found)]


def _exact_dropout(st):
    top = _threshold(st["case"]["p"])

    def some(at, k):
        y = st["x"][at:at + k].double()
        y = y * _exact_kept(st, at, k, y.shape[1]) / (1.0 - top / 2.0 ** 24)
        return [y if st["residual"] is None else y + st["residual"][at:at + k].double()]
    return _in_parts(st, max(1, (1 << 24) // st["x"].shape[1]), some)[0]


def _exact_statistics(s, kind):
    mean = s.sum(1) / s.shape[1] if kind == "layer" else torch.zeros_like(s[:, 0])
    var = ((s - mean[:, None]) ** 2).sum(1) / s.shape[1]
    return (mean if kind == "layer" else None), 1.0 / (var + EPS) ** 0.5


def _exact_seam(st):
    case = st["case"]
    top, hidden = _threshold(case["p"]), case["hidden"]
    one, zero = torch.ones(hidden, dtype=torch.float64, device="cuda"), torch.zeros(hidden, dtype=torch.float64, device="cuda")
    w1, gate, w2 = (one if st[k] is None else st[k].double() for k in ("w1", "gate", "w2"))
    b1, b2 = (zero if st[k] is None else st[k].double() for k in ("b1", "b2"))

    def some(at, k):
        x, (m1, r1, m2, r2) = st["x"][at:at + k].double(), (None,) * 4
        if case["inner"] != "none":
            m1, r1 = _exact_statistics(x, case["inner"])
            x = (x if m1 is None else x - m1[:, None]) * (r1[:, None] * w1) + b1
        x = case["scale"] * gate * x * (_exact_kept(st, at, k, hidden) / (1.0 - top / 2.0 ** 24))
        total = case["residual_scale"] * st["residual"][at:at + k].double() + x
        y = None
        if case["outer"] != "none":
            s = total.to(st["x"].dtype).double()             # the norm is of what the stream holds: rounded to its type
            m2, r2 = _exact_statistics(s, case["outer"])
            y = (s if m2 is None else s - m2[:, None]) * (r2[:, None] * w2) + b2
        return [total, y, m1, r1, m2, r2]
    return dict(zip(("total", "y") + STATS, _in_parts(st, max(1, (1 << 24) // hidden), some)))


def _exact_seam_gradients(st):
    case = st["case"]
    top, hidden = _threshold(case["p"]), case["hidden"]
    one, zero = torch.ones(hidden, dtype=torch.float64, device="cuda"), torch.zeros(hidden, dtype=torch.float64, device="cuda")
    w1, gate, w2 = (one if st[k] is None else st[k].double() for k in ("w1", "gate", "w2"))
    b1 = zero if st["b1"] is None else st["b1"].double()
    m1, r1, m2, r2 = st["stats"].double()[:, :, None]
    sums = {k: zero.clone() for k in ("dw1", "db1", "dgate", "dw2", "db2")}

    def through(d, n, rstd, kind):
        centred = hidden * d - n * (d * n).sum(1, keepdim=True)
        return rstd / hidden * (centred - d.sum(1, keepdim=True) if kind == "layer" else centred)

    def some(at, k):
        rows = slice(at, at + k)
        dt = st["dtotal"][rows].double()
        if case["outer"] != "none":
            dy, n = st["dy"][rows].double(), st["total"][rows].double()
            n = (n - m2[rows] if case["outer"] == "layer" else n) * r2[rows]
            sums["dw2"] += (n * dy).sum(0)
            sums["db2"] += dy.sum(0)
            dt = dt + through(w2 * dy, n, r2[rows], case["outer"])
        g = case["scale"] * dt * _exact_kept(st, at, k, hidden) / (1.0 - top / 2.0 ** 24)
        n = st["x"][rows].double()
        if case["inner"] != "none":
            n = (n - m1[rows] if case["inner"] == "layer" else n) * r1[rows]
        sums["dgate"] += (g * (n * w1 + b1)).sum(0)
        g = gate * g
        sums["dw1"] += (g * n).sum(0)
        sums["db1"] += g.sum(0)
        return [through(w1 * g, n, r1[rows], case["inner"]) if case["inner"] != "none" else g, case["residual_scale"] * dt]
    dx, dresidual = _in_parts(st, max(1, (1 << 24) // hidden), some)
    of = {"dw1": "w1", "db1": "b1", "dgate": "gate", "dw2": "w2", "db2": "b2"}
    return {"dx": dx, "dresidual": dresidual, **{k: v if st[of[k]] is not None else None for k, v in sums.items()}}


def _exact_loss(st):
    case, w = st["case"], st["weight"].double()
    rows = st["x"].shape[0]

    def some(at, k):
        t = st["target"][at:at + k]
        z = st["x"][at:at + k].double() @ w.t()
        lse = torch.logsumexp(z, 1)
        e = case["smoothing"]
        of_target = z[torch.arange(k, device="cuda"), t.clamp(min=0)]
        loss = (1.0 - e) * (lse - of_target) + e * (lse - z.sum(1) / case["vocab"])
        return [loss * (t != IGNORED), lse]
    loss, lse = _in_parts(st, max(1, (1 << 26) // case["vocab"]), some)
    count = max(1, int((st["target"] != IGNORED).sum()))
    return {"loss": loss, "lse": lse, "mean": torch.stack([loss.sum() / count, torch.full((), 1.0 / count, dtype=torch.float64, device="cuda")])}


def _exact_loss_gradients(st):
    case, w = st["case"], st["weight"].double()
    dweight = torch.zeros_like(w)

    def some(at, k):
        x, t = st["x"][at:at + k].double(), st["target"][at:at + k]
        z = x @ w.t()
        soft = torch.exp(z - st["lse"][at:at + k, None].double())
        wanted = torch.full_like(soft, case["smoothing"] / case["vocab"])
        wanted[torch.arange(k, device="cuda"), t.clamp(min=0)] += 1.0 - case["smoothing"]
        d = (soft - wanted) * (st["grad"].double() * st["mean"][1].double() * (t != IGNORED))[:, None]
        dweight.add_(d.t() @ x)
        return [d @ w]
    return {"dx": _in_parts(st, max(1, (1 << 26) // case["vocab"]), some)[0], "dweight": dweight}


def exact(case, seed):
    st = prepare(case, seed)
    return {"dropout": _exact_dropout, "rn_forward": _exact_seam, "rn_backward": _exact_seam_gradients, "ce_forward": _exact_loss,
            "ce_backward": _exact_loss_gradients}[case["path"]](st)


if __name__ == "__main__":
    for c in listed() + [draw(random.Random(k)) for k in range(6)]:
        print(c, work(c))
