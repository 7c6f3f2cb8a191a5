"""The encoder operators at the ends of their arguments' ranges."""
import pytest

from gpu_util import need_cuda

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def ops():
    need_cuda()
    from paper_2608_15438_gb300 import ops as o

    yield o
    o.check(0)


@pytest.mark.parametrize("n", [1, 96, 387, 1536, 5000, 20001])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_an_eps_below_fp32s_range_is_still_positive(ops, n, dtype):
    """Constant rows have no deviation: their norm is the bias for every eps > 0."""
    x = torch.tensor([[0.0], [1.5], [-2.0]], device="cuda").expand(3, n).contiguous().to(dtype)
    b = torch.linspace(-1, 1, n, device="cuda").to(dtype)
    for eps in (1e-5, 1e-40, 1e-46, 1e-60, 1e-300):
        y, mean, rstd = ops.layer_norm(x, None, b, eps=eps, save=True)
        assert torch.equal(y, b.expand(3, n)), eps
        assert torch.equal(mean, x[:, 0].float()) and rstd.isfinite().all()
