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


def test_calls_from_several_threads(ops):
    """Each on a stream of its own, while another thread sets the waits' limit to what it is."""
    import threading

    from paper_2608_15438_gb300 import neuroute as nr

    g = torch.Generator(device="cuda")
    g.manual_seed(11)
    x = torch.randn(600, 256, generator=g, device="cuda").to(BF16)
    w = (torch.randn(512, 256, generator=g, device="cuda") / 16).to(BF16)
    dy = torch.randn(600, 512, generator=g, device="cuda").to(BF16)

    def step():
        h = ops.layer_norm(x)
        y, z = ops.linear(h, w, act="gelu", save="z8")
        return (y,) + ops.linear_backward(dy, h, w, z=z, act="gelu")

    want = step()
    torch.cuda.synchronize()
    wrong, done = [], threading.Event()

    def work():
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            for _ in range(20):
                got = step()
                s.synchronize()
                if not all(torch.equal(a, b) for a, b in zip(got, want)):
                    wrong.append(1)

    def limits():
        while not done.is_set():
            assert nr.lib().nr_ops_wait_limit(0) == 0

    threads = [threading.Thread(target=work) for _ in range(6)]
    other = threading.Thread(target=limits)
    other.start()
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    done.set()
    other.join()
    assert not wrong
    ops.check(0)


def test_empty_batches_in_any_layout(ops):
    """No rows have no strides: slices of a transposed or expanded matrix are taken."""
    w, b = torch.ones(24, 16, device="cuda", dtype=BF16), torch.ones(24, device="cuda")
    x, dy = torch.ones(16, 40, device="cuda", dtype=BF16).T[:0], torch.ones(1, 1, device="cuda", dtype=BF16).expand(0, 24)
    y, z = ops.linear(x, w, b, act="gelu", residual=dy, save="z")
    assert y.shape == z.shape == (0, 24)
    dx, dw, db = ops.linear_backward(dy, x, w, z=dy, act="gelu")
    assert dx.shape == (0, 16) and (dw == 0).all() and (db == 0).all()
    y, mean, rstd = ops.layer_norm(x, save=True)
    dx, dw, db = ops.layer_norm_backward(x, x, None, mean, rstd, residual_grad=x)
    assert y.shape == dx.shape == (0, 16) and (dw == 0).all() and (db == 0).all()
    assert ops.checkpoint8_read(ops.checkpoint8(x)).shape == (0, 16)
    with pytest.raises(ValueError, match="stride"):
        ops.linear(torch.ones(16, 40, device="cuda", dtype=BF16).T, w)
