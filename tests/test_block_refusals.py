"""What dropout's and the residual norm's entry points refuse, on the host and before anything is launched."""
import pytest
import torch

import paper_1908_06077_amd as nuq

EINVAL, ECAPACITY = -1, -2
NAN = float("nan")


def _lib():
    from paper_1908_06077_amd import binding
    return binding._lib


def test_dropout():
    call = _lib().nuq_dropout
    ok = dict(x=16, ldx=8, residual=None, ldr=0, rows=2, hidden=8, type=0, p=0.1, seed=1, step=None, y=16, ldy=8, stream=None)
    assert call(*{**ok, "rows": 0}.values()) == 0 and call(*{**ok, "hidden": 0, "ldy": 0}.values()) == 0      # nothing to do
    for bad in (dict(x=None), dict(x=18), dict(y=None), dict(y=18), dict(ldy=7), dict(residual=18), dict(type=3), dict(p=-0.1),
                dict(p=1.1), dict(p=NAN), dict(step=20), dict(rows=2 ** 31), dict(hidden=2 ** 31), dict(x=17, type=1)):
        assert call(*{**ok, **bad}.values()) == EINVAL, bad


FORWARD = dict(x=16, ldx=8, residual=16, ldr=8, inner=1, w1=None, b1=None, gate=None, outer=1, w2=None, b2=None, rows=2, hidden=8, eps=1e-5,
               scale=1.0, residual_scale=1.0, p=0.1, seed=1, step=None, type=0, weight_type=0, total=16, ldt=8, y=16, ldy=8, stats=16,
               stream=None)
BACKWARD = dict(dy=16, ldg=8, dtotal=16, lda=8, x=16, ldx=8, total=16, ldt=8, inner=1, w1=None, b1=None, gate=None, outer=1, w2=None, rows=2,
                hidden=8, scale=1.0, residual_scale=1.0, p=0.1, seed=1, step=None, type=0, weight_type=0, stats=16, dx=16, ldd=8,
                dresidual=16, lde=8, dw1=16, db1=16, dgate=16, dw2=16, db2=16, workspace=64, bytes=256, stream=None)
BOTH = (dict(x=None), dict(x=18), dict(hidden=0), dict(hidden=16385), dict(rows=2 ** 31), dict(type=3), dict(type=1, weight_type=2),
        dict(inner=3), dict(outer=3), dict(inner=0, outer=0, y=None, dy=None), dict(w1=18), dict(b1=18), dict(gate=18), dict(w2=18),
        dict(scale=NAN), dict(residual_scale=float("inf")), dict(p=-0.1), dict(p=NAN), dict(p=1.01), dict(step=12), dict(stats=18),
        dict(inner=0, w1=16), dict(inner=0, b1=16), dict(type=1, weight_type=1, gate=17))


def test_residual_norm_forward():
    call = _lib().nuq_residual_norm_forward
    assert call(*{**FORWARD, "rows": 0}.values()) == 0                        # nothing to do
    for bad in BOTH + (dict(total=None), dict(total=18), dict(y=None), dict(y=18), dict(ldt=7), dict(ldy=7), dict(residual=18),
                       dict(eps=-1.0), dict(eps=NAN), dict(outer=0), dict(outer=0, y=None, w2=16), dict(outer=0, y=None, b2=16),
                       dict(b2=18)):
        bad = {k: v for k, v in bad.items() if k in FORWARD}
        assert call(*{**FORWARD, **bad}.values()) == EINVAL, bad


def test_residual_norm_backward():
    size = nuq.nuq_residual_norm_workspace_bytes
    assert size(2, 8) == 2 * 8 * 16 and size(10 ** 6, 8) == 1024 * 128 and size(3, 10 ** 4) == 3 * 16 * 10 ** 4 + 24
    call = _lib().nuq_residual_norm_backward
    bare = dict(dw1=None, db1=None, dw2=None, db2=None)
    for bad in BOTH + (dict(dy=None), dict(dy=18), dict(total=None), dict(dx=None), dict(dx=18), dict(ldd=7), dict(lde=7), dict(stats=None),
                       dict(dresidual=18), dict(dw1=18), dict(db1=18), dict(dgate=18), dict(dw2=18), dict(db2=18), dict(workspace=None),
                       dict(workspace=72), dict(dtotal=18), {**bare, "outer": 0}, {**bare, "outer": 0, "dy": None, "dtotal": None},
                       dict(inner=0), dict(outer=0, dy=None)):
        bad = {k: v for k, v in bad.items() if k in BACKWARD}
        assert call(*{**BACKWARD, **bad}.values()) == EINVAL, bad
    wide = dict(hidden=9000, ldg=9000, lda=9000, ldx=9000, ldt=9000, ldd=9000, lde=9000, bytes=10 ** 7, dx=32, dresidual=48)
    for bad in (dict(dx=16), dict(dresidual=16)):                             # the sums of wide rows: not from rows that were replaced
        assert call(*{**BACKWARD, **wide, **bad}.values()) == EINVAL, bad
    assert call(*{**BACKWARD, "bytes": 255}.values()) == ECAPACITY


def test_binding_refuses_tensors_that_do_not_fit(monkeypatch):
    """Host tensors stand in for device tensors: every call here ends in the wrapper."""
    from paper_1908_06077_amd import binding
    monkeypatch.setattr(binding, "_on_device", lambda t: True)
    f = lambda *k: torch.zeros(*k)  # noqa: E731
    i = torch.zeros(1, dtype=torch.int64)

    def forward(x=f(2, 4), residual=None, w1=None, gate=None, w2=None, step=None, total=f(2, 4), y=f(2, 4), stats=f(4, 2)):
        nuq.nuq_residual_norm_forward(x, residual, 1, w1, None, gate, 1, w2, None, 1e-5, 1.0, 1.0, 0.1, 3, step, total, y, stats)

    def backward(dy=f(2, 4), dtotal=None, x=f(2, 4), total=f(2, 4), stats=f(4, 2), dx=f(2, 4), dresidual=None, dgate=None):
        nuq.nuq_residual_norm_backward(dy, dtotal, x, total, 1, None, None, None, 1, None, 1.0, 1.0, 0.1, 3, None, stats, dx, dresidual, None,
                                       None, dgate, None, None, None)
    cases = [
        ("one element or more", lambda: nuq.nuq_dropout(f(2, 0), None, 0.1, 1, None, f(2, 0))),
        ("residual: expected 2 rows", lambda: nuq.nuq_dropout(f(2, 4), f(2, 5), 0.1, 1, None, f(2, 4))),
        ("y: expected dtype", lambda: nuq.nuq_dropout(f(2, 4), None, 0.1, 1, None, f(2, 4).half())),
        ("step: expected dtype", lambda: nuq.nuq_dropout(f(2, 4), None, 0.1, 1, f(1), f(2, 4))),
        ("step holds 0", lambda: nuq.nuq_dropout(f(2, 4), None, 0.1, 1, i[:0], f(2, 4))),
        ("expected float32", lambda: nuq.nuq_dropout(f(2, 4).double(), None, 0.1, 1, i, f(2, 4).double())),
        ("residual: expected dtype", lambda: forward(residual=f(2, 4).half())),
        ("gate holds 3", lambda: forward(gate=f(3))),
        ("weight and bias", lambda: forward(w1=f(4).half())),
        ("outer_weight: expected dtype", lambda: forward(x=f(2, 4).half(), gate=f(4), w2=f(4).half())),
        ("total: expected 2 rows", lambda: forward(total=f(3, 4))),
        ("stats holds", lambda: forward(stats=f(3, 2))),
        ("step: expected dtype", lambda: forward(step=f(1))),
        ("contiguous rows", lambda: forward(y=f(4, 2).t())),
        ("dtotal: expected 2 rows", lambda: backward(dtotal=f(1, 4))),
        ("total: expected dtype", lambda: backward(total=f(2, 4).half())),
        ("stats is needed|stats holds", lambda: backward(stats=f(2, 2))),
        ("dresidual: expected", lambda: backward(dresidual=f(2, 3))),
        ("dgate holds", lambda: backward(dgate=f(5))),
    ]
    for want, call in cases:
        with pytest.raises(ValueError, match=want):
            call()
    monkeypatch.undo()
    with pytest.raises(ValueError, match="device tensor"):
        forward()


LOSS = dict(x=256, ldx=8, weight=256, ldw=8, rows=2, hidden=8, vocab=10, type=0, target=16, ignore=-100, smoothing=0.0)
LOSS_FORWARD = {**LOSS, **dict(loss=None, lse=16, mean=None, workspace=256, bytes=10 ** 6, stream=None)}
LOSS_BACKWARD = {**LOSS, **dict(lse=16, grad=16, per_row=0, mean=None, dx=16, ldd=8, dweight=16, lde=8, workspace=256, bytes=10 ** 9, stream=None)}


def test_linear_cross_entropy():
    size = _lib().nuq_linear_cross_entropy_workspace_bytes
    shape = (256, 64, 256, 64, 100, 64, 1000, 1)
    assert 0 < size(*shape, 0) < size(*shape, 1) < 10 ** 7
    assert size(258, *shape[1:], 0) >= size(*shape, 0) + 100 * 128            # rows that have to be laid out anew
    assert size(*shape[:4], 0, *shape[5:], 1) == 0 and size(*shape[:6], 0, 1, 0) == 0
    forward, backward = _lib().nuq_linear_cross_entropy_forward, _lib().nuq_linear_cross_entropy_backward
    both = (dict(x=None), dict(x=258), dict(weight=None), dict(weight=257), dict(rows=2 ** 20 + 1), dict(hidden=0), dict(hidden=2 ** 16 + 1),
            dict(vocab=0), dict(vocab=2 ** 24 + 1), dict(type=3), dict(target=None), dict(target=20), dict(smoothing=-0.1),
            dict(smoothing=1.0), dict(smoothing=NAN), dict(lse=None), dict(lse=18), dict(mean=18), dict(workspace=None), dict(workspace=264),
            dict(rows=2 ** 20, vocab=2 ** 19))
    for bad in both + (dict(loss=18),):
        assert forward(*{**LOSS_FORWARD, **bad}.values()) == EINVAL, bad
    for bad in both + (dict(grad=None), dict(grad=18), dict(dx=18), dict(dweight=18), dict(ldd=7), dict(lde=7)):
        assert backward(*{**LOSS_BACKWARD, **bad}.values()) == EINVAL, bad


def test_linear_cross_entropy_binding(monkeypatch):
    from paper_1908_06077_amd import binding
    monkeypatch.setattr(binding, "_on_device", lambda t: True)
    f = lambda *k: torch.zeros(*k)  # noqa: E731
    ws, t = torch.zeros(10 ** 6, dtype=torch.uint8), torch.zeros(2, dtype=torch.int64)

    def forward(x=f(2, 4), w=f(9, 4), target=t, loss=None, lse=f(2), mean=None):
        nuq.nuq_linear_cross_entropy_forward(x, w, target, -100, 0.0, loss, lse, mean, ws)

    def backward(grad=f(1), dx=f(2, 4), dw=f(9, 4), lse=f(2)):
        nuq.nuq_linear_cross_entropy_backward(f(2, 4), f(9, 4), t, -100, 0.0, lse, grad, None, dx, dw, ws)
    cases = [
        ("one element or more", lambda: forward(x=f(2, 0), w=f(9, 0))),
        ("rows of the vocabulary", lambda: forward(w=f(9, 2, 4))),
        ("rows of the vocabulary", lambda: forward(w=f(0, 4))),
        ("weight: expected 9 rows of 4", lambda: forward(w=f(9, 5))),
        ("weight: expected dtype", lambda: forward(w=f(9, 4).half())),
        ("target holds 3", lambda: forward(target=torch.zeros(3, dtype=torch.int64))),
        ("target: expected dtype", lambda: forward(target=t.int())),
        ("loss holds 3", lambda: forward(loss=f(3))),
        ("lse holds 1", lambda: forward(lse=f(1))),
        ("mean holds 1", lambda: forward(mean=f(1))),
        ("grad holds 3", lambda: backward(grad=f(3))),
        ("dx: expected 2 rows", lambda: backward(dx=f(2, 5))),
        ("dweight: expected 9 rows", lambda: backward(dw=f(8, 4))),
    ]
    for want, call in cases:
        with pytest.raises(ValueError, match=want):
            call()
