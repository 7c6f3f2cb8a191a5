"""The C entries' refusals of addresses and pitches: codes must lie at 16-byte
addresses wherever a call takes them, other values at multiples of their size,
and no pitch may be negative."""
import pytest

from paper_2608_15438_gb300 import neuroute as nr
from paper_2608_15438_gb300 import ops

P = 1 << 20  # an address that no call gets to
INVALID = -1


def lin(**kw):
    f = dict(m=40, k=64, n=96, dtype=2, y_dtype=2, bias_dtype=0, act=2, x=P, x_ld=64, x_scale=0, x_act=0, w=P,
             w_ld=64, bias=0, residual=0, residual_ld=0, y=P, y_ld=96, z=0, z_ld=0, z_scale=0, dy=P, dy_ld=96,
             dx=P, dx_ld=64, dw=P, dbias=P)
    f.update(kw)
    return ops._LINEAR.pack(*f.values())


def norm(**kw):
    f = dict(m=40, n=96, dtype=2, w_dtype=0, eps=1e-5, x=P, x_ld=0, x_scale=P, weight=0, bias=0, y=P, y_ld=96,
             mean=P, rstd=P, dy=P, dy_ld=96, rg=0, rg_ld=0, dx=P, dx_ld=96, dw=P, db=P)
    f.update(kw)
    return ops._NORM.pack(*f.values())


@pytest.mark.parametrize("off", [1, 2, 4, 8])
@pytest.mark.parametrize("m", [1, 8, 9, 40])
def test_codes_at_other_addresses_are_refused(off, m):
    L = nr.lib()
    a = lin(m=m, z=P + off, z_scale=P)  # z held in 8 bits by the forward call
    assert L.nr_linear_forward_workspace(a, 0) == INVALID
    assert L.nr_linear_forward(a, 0, P, 1 << 40, None) == INVALID
    for kw in (dict(z=P + off, z_scale=P), dict(act=0, x=P + off, x_scale=P),
               dict(z=P, z_scale=P, x=P + off, x_scale=P), dict(act=0, x=P + off, x_scale=P, dw=0)):
        a = lin(m=m, **kw)
        assert L.nr_linear_backward_workspace(a, 0) == INVALID, kw
        assert L.nr_linear_backward(a, 0, P, 1 << 40, None) == INVALID, kw
    assert L.nr_layer_norm_forward(norm(m=m, x=P + off), 0, None) == INVALID
    a = norm(m=m, x=P + off)
    assert L.nr_layer_norm_backward_workspace(a, 0) == INVALID
    assert L.nr_layer_norm_backward(a, 0, P, 1 << 40, None) == INVALID
    assert L.nr_checkpoint8_write(P, 2, m, 32, 32, P + off, P, 0, None) == INVALID
    assert L.nr_checkpoint8_read(P + off, P, m, 32, 0, P, 2, 32, 0, None) == INVALID


def test_values_between_their_types_addresses_are_refused():
    """An address that is no multiple of the element's size, for every matrix and vector."""
    L = nr.lib()
    f32 = dict(y_dtype=0)
    for kw in (dict(x=P + 1), dict(w=P + 1), dict(y=P + 1), dict(residual=P + 1, residual_ld=96), dict(bias=P + 2),
               dict(bias=P + 1, bias_dtype=2), dict(z=P + 1, z_ld=96), dict(y=P + 2, **f32)):
        for m in (1, 40):
            assert L.nr_linear_forward_workspace(lin(m=m, **kw), 0) == INVALID, kw
    for kw in (dict(x=P + 1), dict(w=P + 1), dict(z=P + 1), dict(dy=P + 1), dict(dx=P + 1), dict(dw=P + 1), dict(dbias=P + 2),
               dict(dbias=P + 1, bias_dtype=2), dict(dy=P + 2, **f32)):
        kw = {"z": P, "z_ld": 96, **kw}
        assert L.nr_linear_backward_workspace(lin(**kw), 0) == INVALID, kw
    for kw in (dict(x=P + 1), dict(weight=P + 2), dict(bias=P + 2), dict(y=P + 1), dict(mean=P + 2), dict(rstd=P + 2)):
        assert L.nr_layer_norm_forward(norm(**{"x_scale": 0, "x_ld": 96, **kw}), 0, None) == INVALID, kw
    for kw in (dict(x=P + 1), dict(weight=P + 2), dict(dy=P + 1), dict(rg=P + 1, rg_ld=96), dict(dx=P + 1), dict(mean=P + 2),
               dict(rstd=P + 2), dict(dw=P + 2), dict(db=P + 2)):
        assert L.nr_layer_norm_backward_workspace(norm(**{"x_scale": 0, "x_ld": 96, **kw}), 0) == INVALID, kw
    for dtype, off in ((0, 2), (1, 1), (2, 1)):
        assert L.nr_checkpoint8_write(P + off, dtype, 4, 32, 32, P, P, 0, None) == INVALID
        assert L.nr_checkpoint8_read(P, P, 4, 32, 0, P + off, dtype, 32, 0, None) == INVALID


def test_negative_pitches_are_refused():
    L = nr.lib()
    for kw in (dict(z=P, z_ld=-8), dict(z=P, z_ld=96, x_ld=-1), dict(z=P, z_ld=96, w_ld=-1), dict(z=P, z_ld=96, dy_ld=-96)):
        assert L.nr_linear_backward_workspace(lin(**kw), 0) == INVALID, kw
        assert L.nr_linear_backward(lin(**kw), 0, P, 1 << 40, None) == INVALID, kw
    for kw in (dict(x_scale=0, x_ld=-1), dict(dy_ld=-1), dict(rg=P, rg_ld=-1), dict(dx_ld=-96)):
        assert L.nr_layer_norm_backward_workspace(norm(**kw), 0) == INVALID, kw
    assert L.nr_layer_norm_forward(norm(x_scale=0, x_ld=-1), 0, None) == INVALID
    assert L.nr_checkpoint8_write(P, 2, 4, 32, -1, P, P, 0, None) == INVALID


def test_empty_batches_need_no_addresses():
    """m = 0: nothing is read, so nothing is asked of the pointers."""
    L = nr.lib()
    assert L.nr_linear_forward(lin(m=0, x=0, w=0, y=0, z=1, z_scale=1), 0, None, 0, None) == 0
    assert L.nr_layer_norm_forward(norm(m=0, x=1, y=0), 0, None) == 0
