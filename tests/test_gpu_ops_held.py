"""Layer norms of checkpoints that hold fp16 values near the type's end: past
65504 a held number stands for 65504, in a norm as when it is read back."""
import pytest

from gpu_util import need_cuda

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

F16, F32 = torch.float16, torch.float32


def top_rows(m, n, seed):
    """fp16 rows whose groups of 32 lead with 65504 (64 x 2^10 when held), with
    smaller groups and values of either sign between."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = (torch.rand(m, n, generator=g, device="cuda") * 2 - 0.7) * 48000
    x[torch.rand(m, n, generator=g, device="cuda") < 0.4] = 65504.0
    x[torch.rand(m, n, generator=g, device="cuda") < 0.1] = -65504.0
    x[:, 64:96] *= 2.0 ** -12
    return x.to(F16)


# warps and blocks of every shape, odd widths, and rows read again from memory
@pytest.mark.parametrize("m,n", [(3, 32), (5, 100), (9, 264), (7, 1000), (40, 1536), (6, 2048), (3, 4097), (4, 9000), (2, 20008)])
def test_held_numbers_end_with_the_type(m, n):
    need_cuda()
    from paper_2608_15438_gb300 import ops

    x = top_rows(m, n, n)
    c = ops.checkpoint8(x)
    v = ops.checkpoint8_read(c)  # the values that c stands for
    assert v.isfinite().all() and (v == 65504).any() and (v == -65504).any()
    w = torch.linspace(0.5, 1.5, n, device="cuda")
    y, mean, rstd = ops.layer_norm(c, w, save=True)
    v64 = v.double()
    # (n + 16) 2^-23 of the magnitudes: a sum in fp32 in any order
    assert ((mean.double() - v64.mean(1)).abs() <= (n + 16) * 2.0 ** -23 * v64.abs().mean(1)).all()
    sd = v64.var(1, unbiased=False).add(1e-5).sqrt()
    t = (n + 16) * 2.0 ** -23 * (1 + v64.abs().mean(1) / sd) + 2.0 ** -20
    assert ((rstd.double() * sd - 1).abs() <= t).all()
    # the gradients use the same values: dy of ones in one column, so that dweight is that column's xh
    dy = torch.zeros(m, n, device="cuda", dtype=F16)
    col = int((v == 65504).float().sum(0).argmax())
    dy[:, col] = 1.0
    dx, dw, db = ops.layer_norm_backward(dy, c, w, mean, rstd)
    xh = (v64[:, col] - mean.double()) * rstd.double()
    # xh by one fused operation of terms of up to (|x| + |mean|) rstd
    tol = 2.0 ** -22 * ((v64[:, col].abs() + mean.double().abs()) * rstd.double() + xh.abs()).sum() + m * 2.0 ** -22 * xh.abs().sum()
    assert abs(float(dw[col]) - float(xh.sum())) <= float(tol)
    ops.check(0)


@pytest.mark.parametrize("m,n", [(3, 32), (9, 264), (40, 1536), (6, 2048), (4, 9000), (2, 20008)])
def test_a_held_row_and_its_values_give_the_same_bits(m, n):
    """Where both take one path (aligned widths), also for infinities and NaN."""
    need_cuda()
    from paper_2608_15438_gb300 import ops

    x = top_rows(m, n, n + 1)
    x[0, 5] = float("inf")
    x[1, n - 1] = float("nan")
    c = ops.checkpoint8(x)
    v = ops.checkpoint8_read(c)

    def same(a, b):
        return torch.equal(torch.nan_to_num(a, 1.5, 2.5, -2.5), torch.nan_to_num(b, 1.5, 2.5, -2.5)) and torch.equal(a.isnan(), b.isnan())

    for a, b in zip(ops.layer_norm(c, save=True), ops.layer_norm(v, save=True)):
        assert same(a, b)
    _, mean, rstd = ops.layer_norm(v, save=True)
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    dy = torch.randn(m, n, generator=g, device="cuda").to(F16)
    for a, b in zip(ops.layer_norm_backward(dy, c, None, mean, rstd), ops.layer_norm_backward(dy, v, None, mean, rstd)):
        assert same(a, b)
