"""What the AdamW step passes to the library of a state whose parameters have changed, without a GPU: tensors that say
they are on one, and a stand-in for the library that keeps the table it is given."""
import ctypes
import struct

import pytest
import torch

from paper_2608_15438_gb300 import neuroute as nr
from paper_2608_15438_gb300 import ops, optim

F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


class Library:
    """Keeps the tensors' rows (n, at, p_dtype, g_dtype, decay, p, g) of the last step."""

    def __init__(self):
        self.rows, self.calls = None, 0

    def nr_adamw_step(self, packed, index, ws, nbytes, stream):
        f = ops._ADAMW.unpack(packed)
        count, tensors, p, g = f[:4]
        self.rows = [(*ops._TENSOR.unpack(ctypes.string_at(tensors + i * ops._TENSOR.size, ops._TENSOR.size)),
                      *struct.unpack("q", ctypes.string_at(p + 8 * i, 8)), *struct.unpack("q", ctypes.string_at(g + 8 * i, 8)))
                     for i in range(count)]
        self.calls += 1
        return 0


@pytest.fixture
def library(monkeypatch):
    fake = Library()
    monkeypatch.setattr(nr, "lib", lambda: fake)
    monkeypatch.setattr(ops, "_stream", lambda index: 0)
    monkeypatch.setattr(torch.Tensor, "is_cuda", property(lambda t: True))
    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: 0)
    return fake


def at_the_same_address(p, data):
    address = p.data_ptr()
    p.data = data
    assert p.data_ptr() == address


def test_another_layout_at_the_same_address(library):
    p = torch.nn.Parameter(torch.randn(8, 8))
    s = ops.AdamWState([p])
    ops.adamw_step(s, [torch.ones(8, 8)], 1e-3)
    at_the_same_address(p, p.data.t())
    for _ in range(2):
        with pytest.raises(ValueError, match=r"params\[0\]: changed"):
            ops.adamw_step(s, [torch.ones(8, 8)], 1e-3)
    assert library.calls == 1
    at_the_same_address(p, p.data.t())
    ops.adamw_step(s, [torch.ones(8, 8)], 1e-3)
    assert library.calls == 2
    # the optimizer makes its gradients contiguous, whatever the parameters are
    opt = optim.AdamW([p])
    p.grad = torch.ones(8, 8)
    opt.step()
    at_the_same_address(p, p.data.t())
    p.grad = torch.ones(8, 8).t()
    with pytest.raises(ValueError, match="changed"):
        opt.step()


@pytest.mark.parametrize("shape", [(4, 8), (64,), (32,)])
def test_another_shape_at_the_same_address(library, shape):
    p = torch.nn.Parameter(torch.randn(64)[:32].view(8, 4))
    s = ops.AdamWState([p])
    ops.adamw_step(s, [torch.ones(8, 4)], 1e-3)
    at_the_same_address(p, torch.as_strided(p.data, shape, torch.empty(shape).stride()))
    with pytest.raises(ValueError, match="changed"):
        ops.adamw_step(s, [torch.ones(8, 4)], 1e-3)
    assert library.calls == 1


@pytest.mark.parametrize("old,new", [(F32, BF16), (BF16, F16), (F16, F32)])
def test_another_type_at_the_same_address(library, old, new):
    buf = torch.zeros(64)
    p, q = torch.nn.Parameter(buf.view(old)[:16]), torch.nn.Parameter(torch.zeros(5))
    s = ops.AdamWState([p, q])
    grads = [torch.ones(16), torch.ones(5)]
    for _ in range(2):
        ops.adamw_step(s, grads, 1e-3)
        assert [r[2] for r in library.rows] == [ops._DT[old], ops._DT[F32]]
    at_the_same_address(p, buf.view(new)[:16])
    for _ in range(2):
        ops.adamw_step(s, grads, 1e-3)
        assert [r[:3] for r in library.rows] == [(16, 0, ops._DT[new]), (5, 32, ops._DT[F32])]
        assert [r[5] for r in library.rows] == [p.data_ptr(), q.data_ptr()]


def test_a_device_that_changed(library, monkeypatch):
    p = torch.nn.Parameter(torch.zeros(8))
    s = ops.AdamWState([p])
    ops.adamw_step(s, [torch.ones(8)], 1e-3)
    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: -1 if t is p else 0)
    with pytest.raises(ValueError, match="changed"):
        ops.adamw_step(s, [torch.ones(8)], 1e-3)


def test_parameters_that_came_to_overlap(library):
    buf = torch.zeros(64)
    p, q = torch.nn.Parameter(buf[:32]), torch.nn.Parameter(buf[32:])
    s = ops.AdamWState([p, q])
    grads = [torch.ones(32), torch.ones(32)]
    ops.adamw_step(s, grads, 1e-3)
    q.data = buf[16:48]
    for _ in range(2):
        with pytest.raises(ValueError, match=r"params\[0\] and params\[1\] overlap"):
            ops.adamw_step(s, grads, 1e-3)
    q.data = buf[32:].clone()
    ops.adamw_step(s, grads, 1e-3)
    assert library.calls == 2


def test_a_master_that_was_not_kept_up(library):
    """fp32 values have no master of their own to step: one that becomes 16 bits wide later would be stepped from the
    master of the state's first day."""
    p, q = torch.nn.Parameter(torch.zeros(8)), torch.nn.Parameter(torch.zeros(8, dtype=BF16))
    s = ops.AdamWState([p, q], master=True)
    grads = [torch.ones(8), torch.ones(8)]
    ops.adamw_step(s, grads, 1e-3)
    p.data = p.data.bfloat16()
    for _ in range(2):
        with pytest.raises(ValueError, match=r"params\[0\]: .* master"):
            ops.adamw_step(s, grads, 1e-3)
    p.data = p.data.float()
    ops.adamw_step(s, grads, 1e-3)
    # 16 bits of another kind, and fp32 for 16 bits, which takes no master
    q.data = q.data.half()
    ops.adamw_step(s, grads, 1e-3)
    q.data = q.data.float()
    ops.adamw_step(s, grads, 1e-3)
    q.data = q.data.half()
    with pytest.raises(ValueError, match=r"params\[1\]: .* master"):
        ops.adamw_step(s, grads, 1e-3)
    assert library.calls == 4
    # a refused call leaves nothing behind for the next
    p, q = torch.nn.Parameter(torch.zeros(8, dtype=BF16)), torch.nn.Parameter(torch.zeros(8))
    s = ops.AdamWState([p, q], master=True)
    ops.adamw_step(s, grads, 1e-3)
    want, old = library.rows, (p.data, q.data)
    p.data, q.data = p.data.view(F16), q.data.half()
    with pytest.raises(ValueError, match="master"):
        ops.adamw_step(s, grads, 1e-3)
    p.data, q.data = old
    ops.adamw_step(s, grads, 1e-3)
    assert library.rows == want
    # before the first step the master has the values that the state was made of
    p = torch.nn.Parameter(torch.zeros(8))
    s = ops.AdamWState([p], master=True)
    p.data = p.data.half()
    ops.adamw_step(s, [torch.ones(8)], 1e-3)
    # without masters there is nothing to be out of date
    p = torch.nn.Parameter(torch.zeros(8))
    s = ops.AdamWState([p])
    ops.adamw_step(s, [torch.ones(8)], 1e-3)
    p.data = p.data.half()
    ops.adamw_step(s, [torch.ones(8)], 1e-3)


def test_gradients_that_can_be_read_once(library, monkeypatch):
    """grads and weight_decay as iterators, on the current stream and on another."""
    import contextlib

    monkeypatch.setattr(torch.cuda, "stream", lambda stream: contextlib.nullcontext())
    kept = []
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, stream: kept.append(t.data_ptr()))
    params, grads = [torch.zeros(8), torch.zeros(5)], [torch.ones(8), torch.ones(5)]
    s = ops.AdamWState(params)
    for stream in (None, object()):
        library.rows = None
        ops.adamw_step(s, iter(grads), 1e-3, weight_decay=iter([0.1, 0.2]), stream=stream)
        assert [(r[4], r[6]) for r in library.rows] == [(d, x.data_ptr()) for d, x in zip((0.1, 0.2), grads)]
    assert {t.data_ptr() for t in params + grads} <= set(kept)


def test_arrays_of_a_state_that_overlap(library):
    p = torch.zeros(64)
    flat, step = torch.zeros(128), torch.zeros(1, dtype=torch.int64)
    u8 = torch.zeros(256, dtype=torch.uint8)
    for kw, match in [(dict(m=flat[:64], v=flat[:64]), "m and v"), (dict(m=flat[:64], v=flat[32:96]), "m and v"),
                      (dict(v=p), r"params\[0\] and v"), (dict(master=flat[:64], m=flat[60:124]), "m and master"),
                      (dict(m=flat[:64], step=flat[62:64].view(torch.int64)), "m and step"),
                      (dict(bits=8, m=(u8[:64], u8[64:66]), v=(u8[64:128], u8[200:202])), "m's scales and v"),
                      (dict(bits=8, m=(u8[:64], u8[64:66]), v=(u8[80:144], u8[65:67])), "m's scales and v's scales")]:
        with pytest.raises(ValueError, match=f"{match} overlap"):
            ops.AdamWState([p], **kw)
    s = ops.AdamWState([p], m=flat[:64], v=flat[64:], step=step)
    ops.adamw_step(s, [torch.ones(64)], 1e-3)
    q = torch.nn.Parameter(torch.zeros(64))
    s = ops.AdamWState([q], m=flat[:64], v=flat[64:])
    q.data = flat[:64]
    with pytest.raises(ValueError, match=r"params\[0\] and m overlap"):
        ops.adamw_step(s, [torch.ones(64)], 1e-3)
    ops.AdamWState([torch.zeros(0)], bits=8, m=(u8[:0], u8[:0]), v=(u8[:0], u8[:0]))


def test_gradients_that_are_no_tensors(library):
    import numpy as np

    s = ops.AdamWState([torch.zeros(8), torch.zeros(5)])
    for bad in (np.ones(5, np.float32), [1.0] * 5, 1.0):
        with pytest.raises(TypeError, match=r"grads\[1\]: expected a torch.Tensor"):
            ops.adamw_step(s, [torch.ones(8), bad], 1e-3)
    assert library.calls == 0
    ops.adamw_step(s, [None, torch.ones(5)], 1e-3)
    assert [r[6] != 0 for r in library.rows] == [False, True]
