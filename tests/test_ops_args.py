"""The encoder operators' refusals that need no GPU: the Python checks raise
before the library is called, and the C entries return NR_ERR_INVALID_ARG
before any device work."""
import ctypes
import subprocess

import numpy as np
import pytest
import torch

from paper_2608_15438_gb300 import neuroute as nr
from paper_2608_15438_gb300 import ops

BF16 = torch.bfloat16


@pytest.fixture
def no_library(monkeypatch):
    def called():
        raise AssertionError("the library was called")

    monkeypatch.setattr(nr, "lib", called)


def test_host_tensors_and_wrong_kinds_are_refused(no_library):
    x, w = torch.zeros(4, 16, dtype=BF16), torch.zeros(8, 16, dtype=BF16)
    with pytest.raises(ValueError, match="CUDA"):
        ops.linear(x, w)
    with pytest.raises(ValueError, match="CUDA"):
        ops.linear_backward(torch.zeros(4, 8, dtype=BF16), x, w)
    with pytest.raises(ValueError, match="CUDA"):
        ops.layer_norm(x)
    with pytest.raises(ValueError, match="CUDA"):
        ops.layer_norm_backward(x, x, None, torch.zeros(4), torch.zeros(4))
    with pytest.raises(ValueError, match="CUDA"):
        ops.checkpoint8(x)
    with pytest.raises(ValueError, match="dtype"):
        ops.linear(x.double(), w)
    with pytest.raises(ValueError, match="shape"):
        ops.checkpoint8(x[0])
    with pytest.raises(TypeError):
        ops.layer_norm(np.zeros((4, 16), np.float32))
    with pytest.raises(TypeError):
        ops.checkpoint8_read(x)


def test_structures_have_the_headers_sizes(tmp_path):
    """The packed arguments against the C compiler's layout of the two structures."""
    src = tmp_path / "sizes.c"
    src.write_text('#include <stdio.h>\n#include "neuroute_ops.h"\n'
                   'int main(void) { printf("%zu %zu %zu %zu", sizeof(nr_linear), sizeof(nr_layer_norm),\n'
                   "  __builtin_offsetof(nr_linear, dbias), __builtin_offsetof(nr_layer_norm, eps)); return 0; }\n")
    import os

    inc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
    exe = str(tmp_path / "sizes")
    subprocess.run(["gcc", "-I", inc, "-o", exe, str(src)], check=True)
    got = [int(v) for v in subprocess.run([exe], check=True, capture_output=True, text=True).stdout.split()]
    assert got == [ops._LINEAR.size, ops._NORM.size, ops._LINEAR.size - 8, 32]


def test_c_entries_return_invalid_arg():
    L = nr.lib()

    def lin(**kw):
        f = dict(m=4, k=16, n=8, dtype=2, y_dtype=2, bias_dtype=0, act=0, x=4096, x_ld=16, x_scale=0, x_act=0, w=4096,
                 w_ld=16, bias=0, residual=0, residual_ld=0, y=4096, y_ld=8, z=0, z_ld=0, z_scale=0, dy=0, dy_ld=0,
                 dx=0, dx_ld=0, dw=0, dbias=0)
        f.update(kw)
        return ops._LINEAR.pack(*f.values())

    fwd = [dict(m=-1), dict(k=0), dict(n=0), dict(n=1 << 24), dict(dtype=0), dict(y_dtype=1), dict(act=9), dict(x=0),
           dict(w=0), dict(y=0), dict(y_ld=7), dict(x_ld=-1), dict(x_scale=4096), dict(z=4096, z_ld=4),
           dict(z_scale=4096), dict(bias_dtype=1), dict(m=1 << 31)]
    for kw in fwd:
        assert L.nr_linear_forward_workspace(lin(**kw), 0) < 0, kw
        assert L.nr_linear_forward(lin(**kw), 0, None, 0, None) == -1, kw
    good = dict(dy=4096, dy_ld=8, dx=4096, dx_ld=16)
    for kw in [dict(dy=0), dict(act=2), dict(dx_ld=3), dict(x_act=1), dict(m=1 << 31), dict(dtype=7)]:
        assert L.nr_linear_backward_workspace(lin(**{**good, **kw}), 0) < 0, kw
        assert L.nr_linear_backward(lin(**{**good, **kw}), 0, None, 0, None) == -1, kw

    def norm(**kw):
        f = dict(m=4, n=16, dtype=2, w_dtype=0, eps=1e-5, x=4096, x_ld=16, x_scale=0, weight=0, bias=0, y=4096, y_ld=16,
                 mean=0, rstd=0, dy=0, dy_ld=0, rg=0, rg_ld=0, dx=0, dx_ld=0, dw=0, db=0)
        f.update(kw)
        return ops._NORM.pack(*f.values())

    for kw in [dict(m=-1), dict(n=0), dict(dtype=3), dict(w_dtype=1), dict(eps=0.0), dict(eps=float("nan")), dict(x=0),
               dict(y=0), dict(y_ld=8), dict(mean=4096)]:
        assert L.nr_layer_norm_forward(norm(**kw), 0, None) == -1, kw
    good = dict(dy=4096, dy_ld=16, mean=4096, rstd=4096, dx=4096, dx_ld=16)
    for kw in [dict(dy=0), dict(mean=0), dict(dx=0), dict(dx_ld=2), dict(dw=4096), dict(rg_ld=-1)]:
        assert L.nr_layer_norm_backward_workspace(norm(**{**good, **kw}), 0) < 0, kw
        assert L.nr_layer_norm_backward(norm(**{**good, **kw}), 0, None, 0, None) == -1, kw
    assert L.nr_linear_forward(None, 0, None, 0, None) == -1
    assert L.nr_layer_norm_forward(None, 0, None) == -1
    assert L.nr_checkpoint8_write(None, 0, 4, 16, 16, 4096, 4096, 0, None) == -1
    assert L.nr_checkpoint8_write(4096, 5, 4, 16, 16, 4096, 4096, 0, None) == -1
    assert L.nr_checkpoint8_write(4096, 0, 4, 16, 16, 4097, 4096, 0, None) == -1   # codes misaligned
    assert L.nr_checkpoint8_read(4096, 4096, 4, 16, 9, 4096, 0, 16, 0, None) == -1
    assert L.nr_checkpoint8_read(4096, 4096, 4, 16, 0, 4096, 0, 8, 0, None) == -1
