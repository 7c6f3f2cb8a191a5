"""The block norm around a stream that is far from zero: gradients against the derivative of what forward computed."""
import pytest

from test_gpu_block import BF16, F16, F32, gen, ops  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m,n", [(500, 96), (1000, 387), (300, 1536), (40, 8200)])
@pytest.mark.parametrize("dt,st", [(BF16, BF16), (F16, F16), (BF16, F32), (F32, F32)])
def test_a_stream_with_an_offset(ops, m, n, dt, st):  # noqa: F811
    """A stream far from zero, its deviation small, against the derivative of what forward computed. Backward has y
    as it was stored: half a unit of bf16's last place is a quarter of a deviation there in each yh, and in fp32 2^-18
    of one. The bounds of an fp32 evaluation, begun with a y that is off by its rounding."""
    from bounds import B, near

    g = gen(n)
    r = (100.0 + torch.randn(m, n, generator=g, device="cuda")).to(st)
    u = (0.5 * torch.randn(m, n, generator=g, device="cuda")).to(dt)
    w, b = 1.0 + 0.3 * torch.randn(n, generator=g, device="cuda"), torch.randn(n, generator=g, device="cuda")
    dh = torch.randn(m, n, generator=g, device="cuda").to(dt)
    y, h, stats = ops.block_norm(r, u, pre="layer", weight=w, bias=b, eps=1e-5, save=True)
    d = ops.block_norm_backward(dh, None, y, u, stats, pre="layer", weight=w, bias=b)
    y64 = B(r) + B(u)
    mean = y64.mean()
    dev = y64 - mean
    rstd = (dev * dev).mean().rsqrt(1e-5)
    near(h, dev * rstd * B(w) + B(b), dt, "h")  # from y before its rounding, whatever the stream
    yh = (B(y64.v, y64.tolerance(st)) - mean) * rstd
    q = B(dh) * B(w)
    t = (q - q.mean() - yh * (q * yh).mean()) * rstd
    for got, want, type_, name in ((d.weight, (B(dh) * yh).over(0), F32, "weight"), (d.bias, B(dh).over(0), F32, "bias"),
                                   (d.r, t, st, "r"), (d.u, t, dt, "u")):
        near(got, want, type_, "d" + name)
