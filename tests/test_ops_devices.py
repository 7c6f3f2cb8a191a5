"""The encoder operators asked of a device that is not there: the C entries
return an error before they plan anything. Each case in a process of its own."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEAD = """
from paper_2608_15438_gb300 import neuroute as nr, ops
L = nr.lib()
P = 1 << 20  # an address that no call gets to
def lin(**kw):
    f = dict(m=4, k=16, n=8, dtype=2, y_dtype=2, bias_dtype=0, act=0, x=P, x_ld=16, x_scale=0, x_act=0, w=P,
             w_ld=16, bias=0, residual=0, residual_ld=0, y=P, y_ld=8, z=0, z_ld=0, z_scale=0, dy=P, dy_ld=8,
             dx=0, dx_ld=0, dw=0, dbias=0)
    f.update(kw)
    return ops._LINEAR.pack(*f.values())
def norm(**kw):
    f = dict(m=300, n=387, dtype=2, w_dtype=0, eps=1e-5, x=P, x_ld=387, x_scale=0, weight=0, bias=0, y=P, y_ld=387,
             mean=P, rstd=P, dy=P, dy_ld=387, rg=0, rg_ld=0, dx=P, dx_ld=387, dw=P, db=P)
    f.update(kw)
    return ops._NORM.pack(*f.values())
"""
BOTH = "dx=P, dx_ld=16, dw=P, dbias=P"
CALLS = {
    **{f"forward workspace, {m} rows": f"L.nr_linear_forward_workspace(lin(m={m}), D)" for m in (4, 100, 200, 5000)},
    **{f"backward workspace, {m} rows": f"L.nr_linear_backward_workspace(lin(m={m}, {BOTH}), D)" for m in (1, 9, 200, 5000)},
    "backward workspace, dx": "L.nr_linear_backward_workspace(lin(m=200, dx=P, dx_ld=16), D)",
    "norm workspace": "L.nr_layer_norm_backward_workspace(norm(), D)",
    "norm workspace, long rows": "L.nr_layer_norm_backward_workspace(norm(n=20001, x_ld=20001, dy_ld=20001, dx_ld=20001), D)",
    **{f"forward, {m} rows": f"L.nr_linear_forward(lin(m={m}), D, P, 1 << 40, None)" for m in (4, 200)},
    "backward": f"L.nr_linear_backward(lin(m=200, {BOTH}), D, P, 1 << 40, None)",
    "norm": "L.nr_layer_norm_forward(norm(), D, None)",
    "norm backward": "L.nr_layer_norm_backward(norm(), D, P, 1 << 40, None)",
    "write": "L.nr_checkpoint8_write(P, 2, 4, 32, 32, P, P, D, None)",
    "read": "L.nr_checkpoint8_read(P, P, 4, 32, 0, P, 2, 32, D, None)",
    "status": "L.nr_ops_status(D)",
}


@pytest.mark.parametrize("device", [-1, 64, 99])
def test_a_device_that_is_not_there(device):
    """NR_ERR_CUDA (-5) from every entry, and the process goes on."""
    code = HEAD + f"D = {device}\n" + "".join(f"print(repr({n!r}), {c}, flush=True)\n" for n, c in CALLS.items())
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
    got = dict(line.rsplit(" ", 1) for line in r.stdout.splitlines())
    assert got == {repr(n): "-5" for n in CALLS}


def test_python_names_the_call_and_the_error(monkeypatch):
    from paper_2608_15438_gb300 import neuroute as nr
    from paper_2608_15438_gb300 import ops

    with pytest.raises(nr.NRError, match="nr_linear_forward.*NR_ERR_CUDA"):
        ops._scratch("nr_linear_forward", -5, None)
    with pytest.raises(nr.NRError, match="INVALID_ARG"):
        ops._scratch("nr_linear_forward", -1, None)
