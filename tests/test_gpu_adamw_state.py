"""AdamW states whose parameters become other tensors between steps."""
import pytest

from gpu_util import need_cuda

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


@pytest.fixture
def ops():
    need_cuda()
    from paper_2608_15438_gb300 import ops as o

    return o


@pytest.mark.parametrize("old,new", [(F32, BF16), (BF16, F16), (F16, F32)])
@pytest.mark.parametrize("bits", [32, 8])
def test_another_type_at_the_same_address(ops, old, new, bits):
    """The step is the one that a state over the new tensor takes, and what lies behind it stays."""
    g = torch.Generator(device="cuda").manual_seed(1)
    n = 500
    buf = torch.ones(4 * n, device="cuda")
    p = torch.nn.Parameter(buf.view(old)[:n])
    x = torch.randn(n, generator=g, device="cuda")
    s = ops.AdamWState([p], bits=bits)
    ops.adamw_step(s, [x], 1e-2)
    address = p.data_ptr()
    p.data = buf.view(new)[:n]
    assert p.data_ptr() == address and p.dtype == new
    p.data.copy_(torch.randn(n, generator=g, device="cuda"))
    twin = p.detach().clone()
    t = ops.AdamWState([twin], bits=bits, m=s.m.clone() if bits == 32 else [c.clone() for c in s.m],
                       v=s.v.clone() if bits == 32 else [c.clone() for c in s.v], step=s.step.clone())
    behind = buf.view(new)[n:].clone()
    ops.adamw_step(s, [x], 1e-2)
    ops.adamw_step(t, [x], 1e-2)
    assert torch.equal(p.detach(), twin) and torch.equal(buf.view(new)[n:], behind)


def test_a_transposed_parameter_is_refused(ops):
    from paper_2608_15438_gb300.optim import AdamW

    p = torch.nn.Parameter(torch.randn(64, 64, device="cuda"))
    opt = AdamW([p], lr=1e-2)
    p.grad = torch.ones_like(p)
    opt.step()
    before = p.detach().clone()
    p.data = p.data.t()
    p.grad = torch.randn_like(p)
    with pytest.raises(ValueError, match="does not fit"):
        opt.step()
    assert torch.equal(p.detach(), before.t()) and int(opt.state.step) == 1
