"""Results in the place of the rows they are of: at one stride.  At another, rows that are not read yet would be overwritten; refused on the
host, before anything is launched (no GPU needed)."""
import pytest

from paper_1908_06077_amd import binding

EINVAL, ECAPACITY = -1, -2
DROPOUT = dict(x=1024, ldx=8, residual=2048, ldr=8, rows=2, hidden=8, type=0, p=0.1, seed=1, step=None, y=4096, ldy=8, stream=None)
FORWARD = dict(x=1024, ldx=8, residual=2048, ldr=8, inner=1, w1=None, b1=None, gate=None, outer=1, w2=None, b2=None, rows=2, hidden=8,
               eps=1e-5, scale=1.0, residual_scale=1.0, p=0.1, seed=1, step=None, type=0, weight_type=0, total=4096, ldt=8, y=8192, ldy=8,
               stats=16, stream=None)
BACKWARD = dict(dy=1024, ldg=8, dtotal=2048, lda=8, x=4096, ldx=8, total=8192, ldt=8, inner=1, w1=None, b1=None, gate=None, outer=1, w2=None,
                rows=2, hidden=8, scale=1.0, residual_scale=1.0, p=0.1, seed=1, step=None, type=0, weight_type=0, stats=16, dx=16384, ldd=8,
                dresidual=32768, lde=8, dw1=16, db1=16, dgate=16, dw2=16, db2=16, workspace=64, bytes=100, stream=None)


@pytest.mark.parametrize("call,base,to,ld,of,other", [
    ("nuq_dropout", DROPOUT, "y", "ldy", "x", "ldx"), ("nuq_dropout", DROPOUT, "y", "ldy", "residual", "ldr"),
    ("nuq_residual_norm_forward", FORWARD, "y", "ldy", "x", "ldx"), ("nuq_residual_norm_forward", FORWARD, "total", "ldt", "x", "ldx"),
    ("nuq_residual_norm_forward", FORWARD, "total", "ldt", "residual", "ldr"),
    ("nuq_residual_norm_backward", BACKWARD, "dx", "ldd", "dy", "ldg"), ("nuq_residual_norm_backward", BACKWARD, "dx", "ldd", "x", "ldx"),
    ("nuq_residual_norm_backward", BACKWARD, "dresidual", "lde", "dtotal", "lda"),
    ("nuq_residual_norm_backward", BACKWARD, "dresidual", "lde", "total", "ldt")])
def test_another_stride(call, base, to, ld, of, other):
    f = getattr(binding._lib, call)
    for strides in ({ld: 16}, {other: 16}, {other: 0}, {other: 7}):
        bad = {**base, to: base[of], **strides}
        assert f(*bad.values()) == EINVAL, strides
        if base is BACKWARD:                                  # elsewhere, or of one row, it goes on to the next check
            assert f(*{**base, **strides}.values()) == ECAPACITY and f(*{**bad, "rows": 1}.values()) == ECAPACITY
