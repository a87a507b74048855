"""What the optimizer's and the layer norm's entry points refuse, on the host and before anything is launched."""
import ctypes

import pytest
import torch

import paper_1908_06077_amd as nuq

EINVAL, ECAPACITY = -1, -2


def _lib():
    from paper_1908_06077_amd import binding
    return binding._lib


def _p(*xs):
    return (ctypes.c_void_p * len(xs))(*xs)


def _n(*xs):
    return (ctypes.c_uint64 * len(xs))(*xs)


def _f(*xs):
    return (ctypes.c_float * len(xs))(*xs)


def test_state_blocks():
    assert [nuq.nuq_state_blocks(n) for n in (0, 1, 256, 257, 2 ** 40)] == [0, 1, 1, 2, 2 ** 32]


def test_gradient_norm():
    call = _lib().nuq_gradient_norm
    ok = dict(T=1, g=_p(16), n=_n(4), type=0, max_norm=1.0, workspace=64, bytes=65536, out=16, stream=None)
    for bad in (dict(g=_p(None)), dict(g=_p(18)), dict(type=3), dict(max_norm=0.0), dict(max_norm=-1.0), dict(max_norm=float("nan")),
                dict(workspace=None), dict(workspace=68), dict(bytes=65535), dict(out=None), dict(out=18), dict(g=None), dict(n=None),
                dict(g=_p(17), type=1)):
        assert call(*{**ok, **bad}.values()) == EINVAL, bad


def _steps():
    base = dict(T=1, w=_p(16), g=_p(16), m=_p(16), v=_p(16))
    tail = dict(copy=None, n=_n(4), decay=None, g_type=0, copy_type=1, alpha=0.1, beta1=0.9, beta2=0.99, eps=1e-8, t=1, c=None,
                stream=None)
    return (("nuq_adamw_step", {**base, **tail}), ("nuq_adamw_step_coded", {**base, "scales": _p(16), **tail}))


@pytest.mark.parametrize("which", [0, 1])
def test_adamw(which):
    name, ok = _steps()[which]
    call, nan = getattr(_lib(), name), float("nan")
    cases = [dict(w=_p(None)), dict(w=_p(18)), dict(g=_p(None)), dict(g=_p(18)), dict(m=_p(None)), dict(v=_p(None)), dict(w=None),
             dict(g=None), dict(m=None), dict(v=None), dict(n=None), dict(g_type=3), dict(copy=_p(16), copy_type=0),
             dict(copy=_p(16), copy_type=3), dict(copy=_p(17)), dict(copy=_p(None)), dict(decay=_f(nan)), dict(alpha=nan),
             dict(alpha=float("inf")), dict(beta1=1.0), dict(beta1=-0.1), dict(beta1=nan), dict(beta2=1.0), dict(beta2=nan),
             dict(eps=0.0), dict(eps=-1.0), dict(eps=nan), dict(eps=1e300), dict(t=0), dict(c=18), dict(n=_n(2 ** 63))]
    cases += [dict(scales=_p(None)), dict(scales=_p(18)), dict(scales=None)] if which else [dict(m=_p(18)), dict(v=_p(18))]
    for bad in cases:
        assert call(*{**ok, **bad}.values()) == EINVAL, bad


def test_state_values():
    call = _lib().nuq_adamw_state_values
    assert call(None, None, None, 0, None, None, None) == 0                   # nothing to do
    for k in (0, 1, 2, 4, 5):
        args = [16, 16, 16, 8, 16, 16, None]
        args[k] = None
        assert call(*args) == EINVAL


def test_layer_norm_forward():
    call = _lib().nuq_layer_norm_forward
    ok = dict(x=16, ldx=8, residual=None, ldr=0, weight=None, bias=None, rows=2, hidden=8, eps=1e-5, type=0, weight_type=0, total=None,
              ldt=0, y=16, ldy=8, mean=None, rstd=None, stream=None)
    assert call(*{**ok, "rows": 0}.values()) == 0                             # nothing to do
    for bad in (dict(x=None), dict(x=18), dict(y=None), dict(y=18), dict(ldy=7), dict(residual=16), dict(total=16),
                dict(residual=16, total=16, ldt=7), dict(residual=18, total=16, ldt=8), dict(hidden=0), dict(rows=2 ** 33),
                dict(eps=-1.0), dict(eps=float("nan")), dict(type=3), dict(type=1, weight_type=2), dict(weight=18), dict(bias=18),
                dict(mean=18), dict(rstd=18), dict(type=1, weight_type=1, weight=17)):
        assert call(*{**ok, **bad}.values()) == EINVAL, bad


def test_layer_norm_backward():
    assert nuq.nuq_layer_norm_workspace_bytes(3, 8) == 3 * 8 * 8 and nuq.nuq_layer_norm_workspace_bytes(10 ** 6, 8) == 1024 * 64
    call = _lib().nuq_layer_norm_backward
    ok = dict(dy=16, ldg=8, x=16, ldx=8, weight=None, mean=16, rstd=16, add=None, lda=0, rows=2, hidden=8, type=0, weight_type=0, dx=16,
              ldd=8, dweight=16, dbias=16, workspace=64, bytes=128, stream=None)
    for bad in (dict(dy=None), dict(x=None), dict(dx=None), dict(mean=None), dict(rstd=None), dict(dy=18), dict(ldd=7), dict(add=18),
                dict(dweight=18), dict(dbias=18), dict(weight=18), dict(workspace=None), dict(workspace=72), dict(hidden=0),
                dict(type=3), dict(type=2, weight_type=1), dict(mean=18)):
        assert call(*{**ok, **bad}.values()) == EINVAL, bad
    assert call(*{**ok, "bytes": 127}.values()) == ECAPACITY


def test_binding_refuses_tensors_that_do_not_fit(monkeypatch):
    """Host tensors stand in for device tensors: every call here ends in the wrapper."""
    from paper_1908_06077_amd import binding
    monkeypatch.setattr(binding, "_on_device", lambda t: True)
    f = lambda *k: torch.zeros(*k)  # noqa: E731
    b = lambda k: torch.zeros(k, dtype=torch.uint8)  # noqa: E731
    e = lambda k: b(k).view(torch.float8_e4m3fn)  # noqa: E731
    hyper = (0.1, 0.9, 0.99, 1e-8, 1)
    ws = b(65536)
    norm = nuq.nuq_layer_norm_forward
    back = nuq.nuq_layer_norm_backward
    cases = [
        ("out holds", lambda: nuq.nuq_gradient_norm([f(4)], 1.0, ws, f(1))),
        ("expected dtype", lambda: nuq.nuq_gradient_norm([f(4), f(4).half()], 1.0, ws, f(2))),
        ("expected float32", lambda: nuq.nuq_gradient_norm([f(4).double()], 1.0, ws, f(2))),
        ("contiguous", lambda: nuq.nuq_gradient_norm([f(4, 4).t()[:2]], 1.0, ws, f(2))),
        ("1 tensors, 2 are needed", lambda: nuq.nuq_adamw_step([f(4), f(4)], [f(4)], [f(4)] * 2, [f(4)] * 2, None, *hyper)),
        ("grads.0. holds 3", lambda: nuq.nuq_adamw_step([f(4)], [f(3)], [f(4)], [f(4)], None, *hyper)),
        ("ms.0. holds 5", lambda: nuq.nuq_adamw_step([f(4)], [f(4)], [f(5)], [f(4)], None, *hyper)),
        ("one weight decay", lambda: nuq.nuq_adamw_step([f(4)], [f(4)], [f(4)], [f(4)], [0.1, 0.2], *hyper)),
        ("expected dtype", lambda: nuq.nuq_adamw_step([f(4).half()], [f(4)], [f(4)], [f(4)], None, *hyper)),
        ("copies.0. holds", lambda: nuq.nuq_adamw_step([f(4)], [f(4)], [f(4)], [f(4)], None, *hyper, None, [f(3).half()])),
        ("coefficient holds", lambda: nuq.nuq_adamw_step([f(4)], [f(4)], [f(4)], [f(4)], None, *hyper, f(0))),
        ("scales.0. holds 2", lambda: nuq.nuq_adamw_step_coded([f(257)], [f(257)], [e(257)], [b(257)], [f(2)], None, *hyper)),
        ("expected dtype", lambda: nuq.nuq_adamw_step_coded([f(4)], [f(4)], [b(4)], [b(4)], [f(2)], None, *hyper)),
        ("one length", lambda: nuq.nuq_adamw_state_values(e(4), b(4), f(2), f(4), f(5))),
        ("scales holds", lambda: nuq.nuq_adamw_state_values(e(300), b(300), f(2), f(300), f(300))),
        ("both or neither", lambda: norm(f(2, 4), f(2, 4), None, None, 1e-5, None, f(2, 4), None, None)),
        ("y: expected 2 rows", lambda: norm(f(2, 4), None, None, None, 1e-5, None, f(2, 5), None, None)),
        ("y: expected dtype", lambda: norm(f(2, 4), None, None, None, 1e-5, None, f(2, 4).half(), None, None)),
        ("weight holds", lambda: norm(f(2, 4), None, f(3), None, 1e-5, None, f(2, 4), None, None)),
        ("weight and bias", lambda: norm(f(2, 4).half(), None, f(4).bfloat16(), None, 1e-5, None, f(2, 4).half(), None, None)),
        ("bias: expected dtype", lambda: norm(f(2, 4).half(), None, f(4).half(), f(4), 1e-5, None, f(2, 4).half(), None, None)),
        ("mean holds", lambda: norm(f(2, 4), None, None, None, 1e-5, None, f(2, 4), f(3), None)),
        ("contiguous rows", lambda: norm(f(4, 2).t(), None, None, None, 1e-5, None, f(2, 4), None, None)),
        ("one stride", lambda: norm(f(2, 3, 8)[:, :2, :4], None, None, None, 1e-5, None, f(2, 2, 4), None, None)),
        ("one element or more", lambda: norm(f(2, 0), None, None, None, 1e-5, None, f(2, 0), None, None)),
        ("dy: expected 2 rows", lambda: back(f(3, 4), f(2, 4), None, f(2), f(2), None, f(2, 4), None, None, None)),
        ("rstd holds", lambda: back(f(2, 4), f(2, 4), None, f(2), f(1), None, f(2, 4), None, None, None)),
        ("dbias holds", lambda: back(f(2, 4), f(2, 4), None, f(2), f(2), None, f(2, 4), None, f(5), ws)),
    ]
    for want, call in cases:
        with pytest.raises(ValueError, match=want):
            call()
    monkeypatch.undo()
    with pytest.raises(ValueError, match="device tensor"):
        norm(f(2, 4), None, None, None, 1e-5, None, f(2, 4), None, None)


@pytest.mark.parametrize("which", [0, 1])
def test_adamw_numbers_that_are_none_in_fp32(which):
    name, ok = _steps()[which]
    for bad in (dict(alpha=1e39), dict(alpha=1e38, beta1=0.999), dict(alpha=1e10, decay=_f(3e38))):
        assert getattr(_lib(), name)(*{**ok, **bad}.values()) == EINVAL, bad
