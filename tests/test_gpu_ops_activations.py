"""The activations' stated bounds: values to 2^-20 |z|, slopes to 2^-19, for 16-bit
z over their whole range."""
import pytest

from gpu_util import need_cuda

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from test_gpu_ops import BF16, F16, F32, act64  # noqa: E402


def every(dtype):
    """All finite values of a 16-bit type."""
    v = torch.arange(1 << 16, dtype=torch.int32, device="cuda").to(torch.int16).view(dtype)
    return v[v.isfinite()]


@pytest.mark.parametrize("act", ["gelu", "silu", "relu"])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("rows", [1, 16])
def test_values(act, dtype, rows):
    """z times the unit matrix, in fp32 out; few rows and tensor cores."""
    need_cuda()
    from paper_2608_15438_gb300 import ops

    z = every(dtype)
    z = z[z.abs().float() < 1e37]
    k = 64
    z = torch.nn.functional.pad(z, (0, -z.numel() % (k * rows))).view(-1, rows, k)
    w = torch.eye(k, device="cuda", dtype=dtype)
    worst = 0.0
    for part in z[::1 if rows > 1 else 8]:
        y = ops.linear(part, w, act=act, out_dtype=F32).double()
        z64 = part.double()
        want = torch.where(z64 < -60, 0.0 * z64, act64(z64.clamp(min=-60), act)[0])
        # fp32's own rounding of a value is below 2^-24 |z|; its least number and a flushed one below 2^-126
        off = (y - want).abs() - 2.0 ** -126
        assert (off <= 2.0 ** -20 * z64.abs()).all(), (float(off.max()), act)
        worst = max(worst, float((off / z64.abs().clamp(min=1e-30)).max()))
    print(act, dtype, "worst", worst / 2.0 ** -20, "of the bound")


@pytest.mark.parametrize("act", ["gelu", "silu", "relu"])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_slopes(act, dtype):
    """dbias of one row with dy = 1 is the slope, unrounded."""
    need_cuda()
    from paper_2608_15438_gb300 import ops

    z = every(dtype)[None]
    n = z.shape[1]
    dy = torch.ones(1, n, device="cuda")
    w = torch.zeros(n, 16, device="cuda", dtype=dtype)
    _, _, db = ops.linear_backward(dy, torch.zeros(1, 16, device="cuda", dtype=dtype), w, z=z, act=act, need=(False, False, True))
    z64 = z[0].double()
    want = torch.where(z64 < -60, 0.0 * z64, torch.where(z64 > 60, 1.0 + 0.0 * z64, act64(z64.clamp(-60, 60), act)[1]))
    off = (db.double() - want).abs()
    # GELU: 7.5e-8 of Phi and fp32 roundings of terms of at most 1. SiLU: 1 - s is good to
    # 2^-24 and is multiplied by z, up to 17 where it is not 0 in fp32: 17 2^-24 and as much again
    print(act, dtype, "worst", float(off.max()) / 2.0 ** -19, "of the bound")
    assert (off <= 2.0 ** -19).all(), float(off.max())


def test_gelu_s_lower_tail():
    """What the absolute bound leaves of a small value: under 1e-3 of it at z = -4, 8e-3 at -6."""
    need_cuda()
    from paper_2608_15438_gb300 import ops

    w = torch.eye(16, device="cuda", dtype=BF16)
    for z, bound in ((-1.0, 2e-6), (-2.0, 2e-5), (-4.0, 1e-3), (-6.0, 8e-3)):
        y = float(ops.linear(torch.full((1, 16), z, device="cuda", dtype=BF16), w, act="gelu", out_dtype=F32)[0, 0])
        want = float(act64(torch.tensor(z, dtype=torch.float64), "gelu")[0])
        print("z", z, "relative error", abs(y / want - 1))
        assert abs(y / want - 1) <= bound
